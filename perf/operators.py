"""Dense attention over packed prompts and over a paged key-value cache, and the cache's pages, as cases that can be timed.

Four operators: attention of whole prompts packed one behind the other ("prompt"), attention of one new
token of every sequence over a paged cache ("decode"), making room for new tokens and writing their keys
and values into the pages ("write"), and the life of the pages themselves: sequences forked, others
freed, the rest compacted, with the copies that this takes ("pages"). Sizes are those of the workloads in
``paper_2510_19875_b200/workloads.py`` and of the tests, or plain numbers around them.

With ``own`` the passes go through the public entry points of ``paper_2510_19875_b200.stream``; without it
they are elementary torch operations in fp32, rounded once.
"""
import math
import random

import torch

own = False


def _case(name, kind, **kw):
    return dict(name=name, kind=kind, **kw) if name else dict(kind=kind, **kw)


def _prompt(name, H, G, d, n_seq, longest, lens, *, ahead=0, causal=True, dtype="bf16"):
    """ahead: keys that a sequence has before its first query (a prompt that comes in pieces)."""
    return _case(name, "prompt", H=H, G=G, d=d, n_seq=n_seq, longest=longest, lens=lens, ahead=ahead, causal=causal, dtype=dtype)


def _decode(name, H, G, d, page, n_seq, longest, lens, *, dtype="bf16"):
    return _case(name, "decode", H=H, G=G, d=d, page=page, n_seq=n_seq, longest=longest, lens=lens, dtype=dtype)


def _write(name, G, d, page, n_seq, longest, lens, new, *, dtype="bf16"):
    """new: the most new tokens of a sequence."""
    return _case(name, "write", G=G, d=d, page=page, n_seq=n_seq, longest=longest, lens=lens, new=new, dtype=dtype)


def _pages(name, G, d, page, n_seq, longest, lens, layers, *, dtype="bf16"):
    """n_seq: places for sequences; half of them are taken at first."""
    return _case(name, "pages", G=G, d=d, page=page, n_seq=n_seq, longest=longest, lens=lens, layers=layers, dtype=dtype)


def listed():
    return [
        # a few short questions at once: launches and latency count
        _prompt("prompt_short", 8, 2, 128, 5, 150, 1),
        # one head in fp32, the setting of a first look at one head
        _prompt("prompt_fp32_2k", 1, 1, 64, 1, 2048, 2, dtype="f32"),
        # an ordinary batch of prompts of very different lengths, seven query heads per kv head
        _prompt("prompt_packed", 28, 4, 128, 12, 4500, 3),
        # one long prompt of a GQA layer
        _prompt("prompt_16k", 32, 8, 128, 1, 16384, 4),
        # one short chain of thought: latency
        _decode("decode_one_1k", 32, 8, 128, 64, 1, 1219, 5),
        # a batch of chains of very different lengths
        _decode("decode_batch", 32, 8, 128, 64, 64, 8192, 6),
        # few chains at the longest context: the cache is read once and that is all there is to do
        _decode("decode_128k", 32, 8, 128, 64, 4, 131072, 7),
        # a small model kept in fp32, every head its own keys, small pages
        _decode("decode_fp32", 8, 8, 64, 16, 9, 5003, 8, dtype="f32"),
        # one new token for each of a batch of chains
        _write("write_tokens", 8, 128, 64, 64, 8192, 9, 1),
        # the prompts of a batch
        _write("write_prompts", 8, 128, 64, 24, 8192, 10, 8192),
        # chains of one small layer forked, freed and compacted: launches and latency count
        _pages("pages_one_layer", 2, 64, 16, 16, 500, 11, 1),
        # the same for a stack of layers with a long shared prompt
        _pages("pages_stack", 4, 128, 64, 48, 6000, 12, 28),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = [(32, 8), (28, 4), (8, 2), (12, 2), (16, 16), (6, 2), (1, 1)]


def draw(rng):
    """One more case of the same ranges: lengths log-uniform, from one token on."""
    kind = rng.choice(["prompt", "prompt", "decode", "decode", "write", "pages"])
    H, G = rng.choice(HEADS)
    f32 = rng.random() < 0.2
    dtype = "f32" if f32 else "bf16"
    d = rng.choice([64, 32, 128]) if f32 else rng.choice([128, 128, 128, 64, 64, 256, 32])
    lens = rng.randint(100, 10 ** 6)
    page = rng.choice([16, 32, 64, 64, 128])
    n_seq = _log(rng, 1, 64)
    if kind == "prompt":
        # (a sequence's own square is what costs: the sum of them stays below the largest listed case's)
        most = int(math.sqrt((3.0e8 if f32 else 4.0e9) * 128 / (H * max(d, 64) * max(1, n_seq // 2))))
        longest = _log(rng, 1, min(16384, max(most, 2)))
        ahead = _log(rng, 1, max(longest, 2)) if rng.random() < 0.3 else 0
        return _prompt("", H, G, d, n_seq, max(1, longest - ahead // 2), lens, ahead=ahead // 2, causal=rng.random() < 0.85, dtype=dtype)
    if kind == "decode":
        most = min(131072, int((2 ** 28 if f32 else 2 ** 29) // (n_seq * G * d)))
        return _decode("", H, G, d, page, n_seq, _log(rng, 1, max(most, 2)), lens, dtype=dtype)
    if kind == "write":
        longest = _log(rng, 1, min(32768, 2 ** 28 // (n_seq * G * d)))
        return _write("", G, d, page, n_seq, longest, lens, _log(rng, 1, max(2, longest)), dtype=dtype)
    layers = _log(rng, 1, 28)
    n_seq = max(4, n_seq)
    return _pages("", G, d, page, n_seq, _log(rng, 1, max(2, min(32768, 2 ** 28 // (n_seq * G * d * layers)))), lens, layers, dtype=dtype)


# ------------------------------------------------------------------------------------------------
# Lengths and pages: of the case, whatever the seed
# ------------------------------------------------------------------------------------------------
def _lengths(c):
    """The longest first, the others log-uniform below it; from six sequences on one of them is empty."""
    rng = random.Random(c["lens"])
    lens = [c["longest"]] + [_log(rng, 1, c["longest"]) for _ in range(c["n_seq"] - 1)]
    if c["n_seq"] >= 6:
        lens[4] = 0
    return lens


def _new_tokens(c):
    """How many new tokens each sequence has, its length after them, and the cache's pages: for all of them, and a few to spare."""
    rng = random.Random(c["lens"] + 1)
    lens = _lengths(c)
    new = [min(n, c["new"] if rng.random() < 0.5 else _log(rng, 1, c["new"])) for n in lens]
    return new, lens, sum(-(-n // c["page"]) for n in lens) + 5


def _ledger(c):
    """The pages of the case "pages" before a pass: page table, lengths, how often each page is named, and what
    happens: whose copy each place becomes, and who is done. The even places are taken; every fourth one shares
    its whole pages of the first half with the place four before it. The taken pages lie anywhere in the cache."""
    rng = random.Random(c["lens"] + 2)
    page, n = c["page"], c["n_seq"]
    lens = [m if s % 2 == 0 else 0 for s, m in enumerate(_lengths(c))]
    width = -(-c["longest"] // page) + 1
    n_pages = sum(-(-m // page) for m in lens) * 2 + n + 3
    order = rng.sample(range(n_pages), n_pages)
    table, count = [[-1] * width for _ in range(n)], [0] * n_pages
    for s, m in enumerate(lens):
        shared = min(lens[s - 4] // page, m // page, 1 + m // page // 2) if s >= 4 and s % 4 == 0 else 0
        for j in range(-(-m // page)):
            table[s][j] = table[s - 4][j] if j < shared else order.pop()
            count[table[s][j]] += 1
    parent, done = [-1] * n, [0] * n
    for s in range(1, n, 2):
        if rng.random() < 0.7:
            parent[s] = rng.choice(range(0, n, 4))
    for s in range(2, n, 4):
        done[s] = int(rng.random() < 0.7)
    return table, lens, count, parent, done


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _cu(lens):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return at


def prepare(case, seed):
    c = case
    gen = torch.Generator("cuda").manual_seed(1000003 * seed + 29)
    dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    st = dict(case=c)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    def sink(q, k, first):  # every query looks at its sequence's first key, as trained attention does
        u = normal(k.shape[1], c["d"])
        u /= u.norm(dim=-1, keepdim=True)
        k[first] = 4 * math.sqrt(c["d"]) * u
        q += 2 * u.repeat_interleave(q.shape[1] // k.shape[1], 0)

    if c["kind"] == "prompt":
        lens = _lengths(c)
        keys = [n + c["ahead"] if n else 0 for n in lens]
        q, k, v = normal(sum(lens), c["H"], c["d"]), normal(sum(keys), c["G"], c["d"]), normal(sum(keys), c["G"], c["d"])
        cu = _cu(keys)
        sink(q, k, [a for a, n in zip(cu, keys) if n])
        return dict(st, q=q.to(dt), k=k.to(dt), v=v.to(dt), cu_q=_ints(_cu(lens)), cu_k=_ints(cu))

    page = c["page"]
    if c["kind"] == "pages":
        table, lens, count, parent, done = _ledger(c)
        st.update(table=_ints(table), lens=_ints(lens), count=_ints(count), parent=_ints(parent), done=_ints(done))
        shape = (c["layers"], len(count), page, c["G"], c["d"])
    else:
        lens, new = _lengths(c), [0] * c["n_seq"]
        n_pages = sum(-(-n // page) for n in lens) + 5
        if c["kind"] == "write":
            new, lens, n_pages = _new_tokens(c)
        before = [n - m for n, m in zip(lens, new)]
        width = -(-c["longest"] // page) + 1
        order = random.Random(c["lens"] + 3).sample(range(n_pages), n_pages)
        table = [[order.pop() if j < -(-n // page) else -1 for j in range(width)] for n in before]
        count = [0] * n_pages
        for row in table:
            for x in row:
                if x >= 0:
                    count[x] = 1
        st.update(table=_ints(table), lens=_ints(before), count=_ints(count), new=_ints(new), cu_new=_ints(_cu(new)))
        shape = (1, n_pages, page, c["G"], c["d"])
    st["k_pages"], st["v_pages"] = torch.empty(shape, dtype=dt, device="cuda"), torch.empty(shape, dtype=dt, device="cuda")
    for layer in range(shape[0]):
        st["k_pages"][layer] = normal(*shape[1:])
        st["v_pages"][layer] = normal(*shape[1:])
    if c["kind"] == "decode":
        q = normal(c["n_seq"], c["H"], c["d"])
        first = [row[0] for row in table if row[0] >= 0]
        keys = st["k_pages"][0, :, 0].float()
        sink(q, keys, first)
        st["k_pages"][0, :, 0] = keys.to(dt)
        st["q"] = q.to(dt)
    if c["kind"] == "write":
        st["k_new"], st["v_new"] = normal(sum(new), c["G"], c["d"]).to(dt), normal(sum(new), c["G"], c["d"]).to(dt)
    if c["kind"] != "decode":  # a pass changes the ledger, and starts from this one
        st["ledger"] = [st["table"], st["lens"], st["count"]]
        st["saved"] = [x.clone() for x in st["ledger"]]
    return st


# ------------------------------------------------------------------------------------------------
# One pass
# ------------------------------------------------------------------------------------------------
def run(st):
    kind = st["case"]["kind"]
    if "saved" in st:
        torch._foreach_copy_(st["ledger"], st["saved"])
    if own:
        return _own(st, kind)
    return {"prompt": _plain_prompt, "decode": _plain_decode, "write": _plain_write, "pages": _plain_pages}[kind](st)


def _own(st, kind):
    from paper_2510_19875_b200 import stream as S

    if kind == "prompt":
        return S.prompt_attention(st["q"], st["k"], st["v"], st["cu_q"], st["cu_k"], causal=st["case"]["causal"], want_lse=True)
    if "cache" not in st:  # the handle that a program keeps with its cache
        st["cache"] = S.PagedCache(st["k_pages"], st["v_pages"], st["table"], st["lens"], st["count"])
    cache = st["cache"]
    if kind == "decode":
        return S.decode_attention(st["q"], cache, want_lse=True)
    if kind == "write":
        info = S.cache_reserve(cache, st["new"])
        S.cache_write(cache, st["k_new"], st["v_new"], st["cu_new"], info=info)
        return info, *st["ledger"], cache.k, cache.v
    forked = S.cache_fork(cache, st["parent"])
    S.cache_copy_pages(cache, forked)
    freed = S.cache_free(cache, st["done"])
    packed = S.cache_compact(cache)
    S.cache_copy_pages(cache, packed)
    return forked.pairs, forked.info, freed, packed.pairs, packed.info, *st["ledger"], cache.k, cache.v


def _softmax_product(scores, v, how):
    """exp(scores) v over the last axis, divided by its sum; rows without a finite score give zeros and -inf."""
    top = scores.amax(-1, keepdim=True)
    shift = torch.where(top > -math.inf, top, 0.0)
    weights = torch.exp(scores - shift)
    total = weights.sum(-1)
    out = torch.einsum(how, weights, v) / torch.where(total > 0, total, 1.0).unsqueeze(-1)
    return out, shift.squeeze(-1) + torch.log(total)


def _plain_prompt(st):
    """All sequences at once, padded to the longest; some kv heads at a time where the scores would not fit."""
    c, q, k, v, cu_q, cu_k = (st[n] for n in ("case", "q", "k", "v", "cu_q", "cu_k"))
    H, G, d = c["H"], c["G"], c["d"]
    n_q, n_k = c["longest"], c["longest"] + c["ahead"]
    lens_q, lens_k = cu_q.diff(), cu_k.diff()
    i, j = torch.arange(n_q, device="cuda"), torch.arange(n_k, device="cuda")
    at_q, at_k = cu_q[:-1, None] + i, cu_k[:-1, None] + j
    there_q, there_k = i < lens_q[:, None], j < lens_k[:, None]
    allowed = there_q[:, :, None] & there_k[:, None, :]
    if c["causal"]:  # the last query sees every key
        allowed = allowed & (j <= i[:, None] + (lens_k - lens_q)[:, None, None])
    N = q.shape[0]
    rows, keys = at_q.clamp(max=N - 1), at_k.clamp(max=k.shape[0] - 1)
    out, lse = torch.empty(N, H, d, device="cuda"), torch.empty(H, N, device="cuda")
    place = torch.where(there_q, at_q, N).view(-1)  # (what pads goes behind the end)
    step = max(1, min(G, int(2 ** 32 // (c["n_seq"] * n_q * n_k * (H // G)))))
    for g in range(0, G, step):
        e = min(G, g + step)
        a, b = g * (H // G), e * (H // G)
        qs = q[rows][:, :, a:b].float().view(c["n_seq"], n_q, e - g, H // G, d)
        ks, vs = k[keys][:, :, g:e].float(), v[keys][:, :, g:e].float()
        scores = torch.einsum("sighd,sjgd->sghij", qs, ks) / math.sqrt(d)
        scores.masked_fill_(~allowed[:, None, None], -math.inf)
        o, ls = _softmax_product(scores, vs, "sghij,sjgd->sghid")
        o = o.permute(0, 3, 1, 2, 4).reshape(-1, b - a, d)
        ls = ls.permute(1, 2, 0, 3).reshape(b - a, -1)
        out[:, a:b] = torch.empty(N + 1, b - a, d, device="cuda").index_copy_(0, place, o)[:N]
        lse[a:b] = torch.empty(b - a, N + 1, device="cuda").index_copy_(1, place, ls)[:, :N]
    return out.to(q.dtype), lse


def _plain_decode(st):
    c, q, table, lens = (st[n] for n in ("case", "q", "table", "lens"))
    n, width = table.shape
    pages = table.clamp(min=0)
    k, v = (st[x][0][pages].view(n, width * c["page"], c["G"], c["d"]).float() for x in ("k_pages", "v_pages"))
    there = torch.arange(width * c["page"], device="cuda") < lens[:, None]
    v = torch.where(there[:, :, None, None], v, 0.0)
    scores = torch.einsum("sghd,sjgd->sghj", q.float().view(n, c["G"], -1, c["d"]), k) / math.sqrt(c["d"])
    scores.masked_fill_(~there[:, None, None], -math.inf)
    out, lse = _softmax_product(scores, v, "sghj,sjgd->sghd")
    return out.reshape(q.shape).to(q.dtype), lse.reshape(n, c["H"])


def _info(done, moved, free, bad):
    return torch.stack([done, moved, free, bad]).to(torch.int32)


def _free_pages(count):
    """The free pages in ascending order (behind them the others), and how many there are."""
    free = count == 0
    at = torch.arange(count.numel(), device="cuda")
    return torch.sort(torch.where(free, at, at + count.numel())).values % count.numel(), free.sum()


def _take(count, free, n_taken):
    """The n_taken lowest free pages are named once."""
    taken = (count == 0) & ((count == 0).cumsum(0) <= n_taken)
    count.copy_(torch.where(taken, 1, count))


def _plain_write(st):
    c, (table, lens, count), new, cu = st["case"], st["ledger"], st["new"], st["cu_new"]
    page, width = c["page"], table.shape[1]
    free, n_free = _free_pages(count)
    have, after = -(-lens // page), -(-(lens + new) // page)
    bad = ((new < 0) | (after > width)).sum()
    need = after - have
    total = need.sum()
    done = (bad == 0) & (total <= n_free)
    j = torch.arange(width, device="cuda")
    fresh = done & (j >= have[:, None]) & (j < after[:, None])
    which = (need.cumsum(0) - need)[:, None] + j - have[:, None]
    table.copy_(torch.where(fresh, free[which.clamp(0, free.numel() - 1)], table))
    taken = torch.where(done, total, 0)
    _take(count, free, taken)
    lens.copy_(torch.where(done, lens + new, lens))
    n = st["k_new"].shape[0]
    token = torch.arange(n, device="cuda", dtype=torch.int32)
    slot = torch.searchsorted(cu, token, right=True) - 1
    pos = lens[slot] - new[slot] + token - cu[slot]
    to = table[slot, pos // page], pos % page
    st["k_pages"][0].index_put_(to, st["k_new"])
    st["v_pages"][0].index_put_(to, st["v_new"])
    return _info(done, torch.where(done, total, total), n_free - taken, bad), table, lens, count, st["k_pages"], st["v_pages"]


def _copy_pages(st, pairs):
    pairs = pairs[pairs[:, 0] >= 0]
    for x in (st["k_pages"], st["v_pages"]):
        x[:, pairs[:, 1]] = x[:, pairs[:, 0]]


def _plain_pages(st):
    c, (table, lens, count), parent, ends = st["case"], st["ledger"], st["parent"], st["done"]
    page, (n, width), n_pages = c["page"], table.shape, count.numel()
    j, at = torch.arange(width, device="cuda"), torch.arange(n_pages, device="cuda")
    zero = torch.zeros((), dtype=torch.int64, device="cuda")
    # fork: whole pages are shared, one that is not full is copied
    child = parent >= 0
    src = parent.clamp(min=0)
    free, n_free = _free_pages(count)
    n_src = torch.where(child, lens[src], 0)
    partial = n_src % page != 0
    place = partial.cumsum(0) - 1
    fresh = free[place.clamp(min=0)]
    here = child[:, None] & (j < -(-n_src // page)[:, None])
    last = partial[:, None] & (j == (n_src // page)[:, None])
    of_src = table[src]
    from_page = torch.where(last, of_src, 0).sum(1)
    pairs = torch.full((n + 1, 2), -1, dtype=torch.int32, device="cuda")
    pairs[torch.where(partial, place, n)] = torch.where(partial[:, None], torch.stack([from_page, fresh], 1), -1).to(torch.int32)
    pairs = pairs[:n].contiguous()
    table.copy_(torch.where(last, fresh[:, None], torch.where(here, of_src, table)))
    lens.copy_(torch.where(child, n_src, lens))
    count.index_add_(0, table.clamp(min=0).view(-1), here.view(-1).to(torch.int32))
    forked = _info(zero + 1, partial.sum(), (count == 0).sum(), zero)
    _copy_pages(st, pairs)
    # free
    gone = (ends != 0)[:, None] & (j < -(-lens // page)[:, None])
    n_free = (count == 0).sum()
    count.index_add_(0, table.clamp(min=0).view(-1), -gone.view(-1).to(torch.int32))
    table.masked_fill_((ends != 0)[:, None], -1)
    lens.masked_fill_(ends != 0, 0)
    freed = _info(zero + 1, (count == 0).sum() - n_free, (count == 0).sum(), zero)
    # compact: the used pages beyond the number of used pages go to the free ones below it, both in ascending order
    used = count > 0
    n_used = used.sum()
    mover, hole = used & (at >= n_used), ~used & (at < n_used)
    movers, holes = (torch.sort(torch.where(x, at, n_pages)).values for x in (mover, hole))
    remap = torch.cat([at, at[-1:] + 1]).index_copy_(0, movers, holes)[:n_pages]
    back = torch.cat([at, at[-1:] + 1]).index_copy_(0, holes, movers)[:n_pages]
    moves = torch.stack([movers, holes], 1)[: n_pages // 2].to(torch.int32)
    moves = torch.where(moves < n_pages, moves, -1)
    table.copy_(torch.where(table >= 0, remap[table.clamp(min=0)], table))
    count.copy_(torch.where(at < n_used, count[back.clamp(max=n_pages - 1)], 0))
    packed = _info(zero + 1, mover.sum(), n_pages - n_used, zero)
    _copy_pages(st, moves)
    return pairs, forked, freed, moves, packed, table, lens, count, st["k_pages"], st["v_pages"]


# ------------------------------------------------------------------------------------------------
def work(case):
    c = case
    e = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "prompt":
        lens = _lengths(c)
        keys = [n + c["ahead"] if n else 0 for n in lens]
        pairs = sum(n * m - (n * (n - 1) // 2 if c["causal"] else 0) for n, m in zip(lens, keys))
        n, m = sum(lens), sum(keys)
        return {"bytes": 2.0 * e * c["d"] * (n * c["H"] + m * c["G"]) + 4.0 * n * c["H"], "flops": 4.0 * c["d"] * c["H"] * pairs}
    page = c["page"]
    if c["kind"] == "decode":
        lens = _lengths(c)
        ledger = 4.0 * (len(lens) + sum(-(-n // page) for n in lens))
        return {"bytes": 2.0 * e * c["d"] * (sum(lens) * c["G"] + len(lens) * c["H"]) + 4.0 * len(lens) * c["H"] + ledger,
                "flops": 4.0 * c["d"] * c["H"] * sum(lens)}
    if c["kind"] == "write":  # read and written once; which pages are free, and the table's new entries
        new, _, n_pages = _new_tokens(c)
        return {"bytes": 4.0 * e * c["d"] * c["G"] * sum(new) + 4.0 * (n_pages + 4 * c["n_seq"]), "flops": 0.0}
    table, lens, count, _, _ = _ledger(c)
    pairs, _, _, moves, _, _, _, _ = _lives(c)
    copies = sum(p[0] >= 0 for p in pairs) + sum(p[0] >= 0 for p in moves)
    entries = sum(-(-n // page) for n in lens)
    return {"bytes": 4.0 * e * c["layers"] * page * c["G"] * c["d"] * copies + 4.0 * (6 * len(count) + 4 * entries + 8 * copies), "flops": 0.0}


def _lives(c):
    """The pages' lives step by step, in whole numbers: what a pass of "pages" leaves of the ledger."""
    table, lens, count, parent, done = _ledger(c)
    page, n_pages = c["page"], len(count)
    heap = [p for p in range(n_pages) if count[p] == 0]
    pairs = []
    for s, f in enumerate(parent):
        if f < 0:
            continue
        lens[s] = lens[f]
        for x in range(-(-lens[f] // page)):
            if (x + 1) * page <= lens[f]:
                table[s][x] = table[f][x]
            else:
                table[s][x] = heap.pop(0)
                pairs.append([table[f][x], table[s][x]])
            count[table[s][x]] += 1
    forked = [1, len(pairs), count.count(0), 0]
    before = count.count(0)
    for s, x in enumerate(done):
        if x:
            for y in table[s]:
                if y >= 0:
                    count[y] -= 1
            table[s], lens[s] = [-1] * len(table[s]), 0
    freed = [1, count.count(0) - before, count.count(0), 0]
    n_used = n_pages - count.count(0)
    moves = list(map(list, zip([p for p in range(n_used, n_pages) if count[p]], [p for p in range(n_used) if not count[p]])))
    to = dict(moves)
    table = [[to.get(x, x) for x in row] for row in table]
    for a, b in moves:
        count[b], count[a] = count[a], 0
    packed = [1, len(moves), n_pages - n_used, 0]
    pairs += [[-1, -1]] * (c["n_seq"] - len(pairs))
    moves += [[-1, -1]] * (n_pages // 2 - len(moves))
    return pairs, forked, freed, moves, packed, table, lens, count


def _exact_attention(q, k, v, first):
    """q [n, H, d], k and v [m, G, d] in 64 bits, query i sees the keys up to first + i (all of them if first is None)."""
    n, H, d = q.shape
    m, G = k.shape[:2]
    out, lse = torch.zeros(n, H, d, dtype=torch.float64, device="cuda"), torch.full((H, n), -math.inf, dtype=torch.float64, device="cuda")
    if m == 0 or n == 0:
        return out, lse
    for h in range(H):
        s = (q[:, h].double() @ k[:, h * G // H].double().T) * d ** -0.5
        if first is not None:
            hidden = torch.arange(m, device="cuda")[None] > torch.arange(n, device="cuda")[:, None] + first
            s.masked_fill_(hidden, -math.inf)
        lse[h] = torch.logsumexp(s, 1)
        p = torch.exp(s - torch.where(lse[h] > -math.inf, lse[h], 0.0)[:, None])
        out[:, h] = p @ v[:, h * G // H].double()
    return out, lse


def exact(case, seed):
    c = case
    st = prepare(case, seed)
    if c["kind"] == "prompt":
        parts = []
        for s in range(c["n_seq"]):
            a, b, x, y = (int(t) for t in (st["cu_q"][s], st["cu_q"][s + 1], st["cu_k"][s], st["cu_k"][s + 1]))
            parts.append(_exact_attention(st["q"][a:b], st["k"][x:y], st["v"][x:y], (y - x) - (b - a) if c["causal"] else None))
        return torch.cat([o for o, _ in parts]), torch.cat([x for _, x in parts], 1)
    if c["kind"] == "decode":
        parts = []
        for s in range(c["n_seq"]):
            n = int(st["lens"][s])
            pages = st["table"][s, : -(-n // c["page"])].long()
            k, v = (st[x][0][pages].view(-1, c["G"], c["d"])[:n] for x in ("k_pages", "v_pages"))
            parts.append(_exact_attention(st["q"][s:s + 1], k, v, None))
        return torch.cat([o for o, _ in parts]), torch.cat([x.T for _, x in parts])
    k, v = st["k_pages"], st["v_pages"]
    if c["kind"] == "write":
        page = c["page"]
        new, after, n_pages = _new_tokens(c)
        table, count = st["table"].tolist(), st["count"].tolist()
        heap, taken, at = [p for p in range(n_pages) if count[p] == 0], 0, 0
        places = []
        for s, n in enumerate(after):
            for x in range(-(-(n - new[s]) // page), -(-n // page)):
                table[s][x] = heap.pop(0)
                count[table[s][x]] = 1
                taken += 1
            places += [table[s][p // page] * page + p % page for p in range(n - new[s], n)]
        where = torch.tensor(places, dtype=torch.int64, device="cuda")
        for x, y in ((k, st["k_new"]), (v, st["v_new"])):
            x.view(n_pages * page, c["G"], c["d"])[where] = y
        return _ints([1, taken, len(heap), 0]), _ints(table), _ints(after), _ints(count), k, v
    pairs, forked, freed, moves, packed, table, lens, count = _lives(c)
    from_page = list(range(len(count)))  # whose first content a page holds at the end
    for a, b in pairs + moves:
        if a >= 0:
            from_page[b] = from_page[a]
    order = torch.tensor(from_page, device="cuda")
    for x in (k, v):
        for layer in range(c["layers"]):
            x[layer] = x[layer][order]
    return _ints(pairs), _ints(forked), _ints(freed), _ints(moves), _ints(packed), _ints(table), _ints(lens), _ints(count), k, v
