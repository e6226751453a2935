"""Attention with a sliding window and sinks, and the paged cache in 8 bits, as cases that can be timed.

Four passes: attention of packed prompts whose queries see the last ``window`` keys and the first ``sinks`` ones
("window"), the same for one new token of every sequence over a paged cache ("window_decode"), making room for new
tokens in a cache of 8 bits, writing them and reading sequences back as a prompt that comes in pieces needs them
("write8"), and attention of one new token of every sequence over such a cache ("decode8"). Sizes are those of the
workloads in ``paper_2510_19875_b200/workloads.py`` and of the tests, or plain numbers around them.

The cache of 8 bits holds e4m3 numbers and for every block of tokens, kv head, keys and values a scale: the smallest power of
two 2^e, -90 <= e <= 120, with no element beyond 448 2^e. A block that has tokens and gets more keeps its scale or
takes the new ones', whichever is larger, and what it holds is rounded again where the scale grows.

With ``own`` the passes go through the public entry points of ``paper_2510_19875_b200.stream``; without it
they are elementary torch operations in fp32, rounded once.
"""
import math
import random

import torch

own = False

E4M3 = torch.float8_e4m3fn


def _case(name, kind, **kw):
    return dict(name=name, kind=kind, **kw) if name else dict(kind=kind, **kw)


def _window(name, H, G, d, n_seq, longest, lens, window, sinks, *, ahead=0, dtype="bf16"):
    """ahead: keys that a sequence has before its first query (a prompt that comes in pieces)."""
    return _case(name, "window", H=H, G=G, d=d, n_seq=n_seq, longest=longest, lens=lens, window=window, sinks=sinks, ahead=ahead, dtype=dtype)


def _window_decode(name, H, G, d, page, n_seq, longest, lens, window, sinks, *, dtype="bf16"):
    return _case(name, "window_decode", H=H, G=G, d=d, page=page, n_seq=n_seq, longest=longest, lens=lens, window=window, sinks=sinks, dtype=dtype)


def _write8(name, G, d, page, block, n_seq, longest, lens, new, *, whole=True, dtype="bf16"):
    """new: the most new tokens of a sequence. Whole sequences are read back, or what lies in blocks that have new tokens."""
    return _case(name, "write8", G=G, d=d, page=page, block=block, n_seq=n_seq, longest=longest, lens=lens, new=new, whole=whole, dtype=dtype)


def _decode8(name, H, G, d, page, block, n_seq, longest, lens, *, window=0, sinks=0, dtype="bf16"):
    """window 0: every key is seen."""
    return _case(name, "decode8", H=H, G=G, d=d, page=page, block=block, n_seq=n_seq, longest=longest, lens=lens, window=window, sinks=sinks, dtype=dtype)


def listed():
    return [
        # a few short questions at once, most of them longer than the window: launches and latency count
        _window("window_short", 8, 2, 128, 5, 150, 1, 64, 4),
        # one head in fp32, the setting of a first look at one head
        _window("window_fp32_2k", 1, 1, 64, 1, 2048, 2, 256, 4, dtype="f32"),
        # an ordinary batch of prompts of very different lengths, seven query heads per kv head
        _window("window_packed", 28, 4, 128, 12, 4500, 3, 1024, 4),
        # one long prompt of a GQA layer, a window of the length that long contexts are run with
        _window("window_32k", 32, 8, 128, 1, 32768, 4, 4096, 16),
        # a batch of chains of very different lengths, some of them shorter than the window
        _window_decode("window_decode_batch", 32, 8, 128, 64, 64, 8192, 6, 1024, 4),
        # few chains at the longest context, which all have far more tokens than they look at, in fp32 with small pages
        _window_decode("window_decode_fp32", 8, 8, 64, 16, 9, 50003, 8, 1000, 3, dtype="f32"),
        # one new token for each of a batch of chains: most blocks have some already
        _write8("write8_tokens", 8, 128, 64, 64, 64, 8192, 9, 1, whole=False),
        # the prompts of a batch, or the rest of them, and what attention needs of it
        _write8("write8_prompts", 8, 128, 64, 64, 24, 8192, 10, 8192),
        # one short chain of thought: latency
        _decode8("decode8_one_1k", 32, 8, 128, 64, 64, 1, 1219, 5),
        # a batch of chains of very different lengths, a scale for 16 tokens
        _decode8("decode8_batch", 32, 8, 128, 64, 16, 64, 8192, 6),
        # few chains at the longest context: the cache is read once and that is all there is to do
        _decode8("decode8_128k", 32, 8, 128, 64, 64, 4, 131072, 7),
        # a small model kept in fp32 but for its cache, every head its own keys, small pages, a window
        _decode8("decode8_fp32", 8, 8, 64, 16, 16, 9, 5003, 8, window=2500, sinks=7, dtype="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(hi, lo))))))


HEADS = [(32, 8), (28, 4), (8, 2), (12, 2), (16, 16), (6, 2), (1, 1)]


def draw(rng):
    """One more case of the same ranges: lengths and windows log-uniform, from one token on."""
    kind = rng.choice(["window", "window", "window_decode", "write8", "decode8", "decode8"])
    H, G = rng.choice(HEADS)
    f32 = rng.random() < 0.2
    dtype = "f32" if f32 else "bf16"
    d = rng.choice([64, 32, 128]) if f32 else rng.choice([128, 128, 128, 64, 64, 256, 32])
    lens = rng.randint(100, 10 ** 6)
    page, block = rng.choice([(16, 16), (32, 16), (64, 64), (64, 16), (64, 32), (128, 128), (24, 8)])
    n_seq = _log(rng, 1, 64)
    sinks = rng.choice([0, 1, 4, 16, _log(rng, 1, 300)])
    if kind == "window":
        # (pairs of a query and a key are what costs: the sum of them stays below the largest listed case's)
        longest = _log(rng, 1, min(32768, 2 ** 26 // (H * max(d, 64) * max(1, n_seq // 2))))
        most = (1.0e8 if f32 else 4.0e9) * 128 / (H * max(d, 64) * max(1, n_seq // 2) * longest)
        window = _log(rng, 1, max(2, int(min(most, 2 * longest))))
        ahead = _log(rng, 1, max(longest, 2)) if rng.random() < 0.3 else 0
        return _window("", H, G, d, n_seq, max(1, longest - ahead // 2), lens, window, sinks, ahead=ahead // 2, dtype=dtype)
    if kind == "window_decode":
        longest = _log(rng, 1, max(2, min(131072, int((2 ** 28 if f32 else 2 ** 29) // (n_seq * G * d)))))
        return _window_decode("", H, G, d, page, n_seq, longest, lens, _log(rng, 1, 2 * longest), sinks, dtype=dtype)
    if kind == "decode8":
        longest = _log(rng, 1, max(2, min(131072, int((2 ** 28 if f32 else 2 ** 29) // (n_seq * G * d)))))
        window = _log(rng, 1, longest) if rng.random() < 0.3 else 0
        return _decode8("", H, G, d, page, block, n_seq, longest, lens, window=window, sinks=sinks if window else 0, dtype=dtype)
    longest = _log(rng, 1, max(2, min(32768, 2 ** 27 // (n_seq * G * d))))
    return _write8("", G, d, page, block, n_seq, longest, lens, _log(rng, 1, max(2, longest)), whole=rng.random() < 0.7, dtype=dtype)


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
    """How many new tokens each sequence has: all of them, or a part."""
    rng = random.Random(c["lens"] + 1)
    return [min(n, c["new"] if rng.random() < 0.5 else _log(rng, 1, c["new"])) for n in _lengths(c)]


def _read_back(c):
    """How many tokens of each sequence are read back."""
    return [n if c["whole"] else n - (n - m) // c["block"] * c["block"] for n, m in zip(_lengths(c), _new_tokens(c))]


def _table(c, lens, n_pages):
    """Pages anywhere in the cache for the tokens that there are, and the rest of them in the order they would be taken."""
    order = random.Random(c["lens"] + 3).sample(range(n_pages), n_pages)
    width = -(-c["longest"] // c["page"]) + 1
    return [[order.pop() if j < -(-n // c["page"]) else -1 for j in range(width)] for n in lens]


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _cu(lens):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return at


def _two_to(e):
    """2^e for whole numbers, exact, in 64 bits."""
    return (e.long() + 1023 << 52).view(torch.float64)


def _scales_of(top):
    """The smallest power of two 2^e, -90 <= e <= 120, with top <= 448 2^e (top: fp32)."""
    part, e = torch.frexp(top)  # (top = part 2^e, 0.5 <= part < 1; 448 = 0.875 2^9)
    e = (e - 9 + (part > 0.875).to(e.dtype)).clamp(-90, 120)
    return _two_to(torch.where(top > 0, e, -90)).float()


def _fill8(st, c, n_pages, normal):
    """Pages full of e4m3 numbers and their scales. Some channels of the keys stand out, as trained models' do, and blocks differ in size."""
    bpp = c["page"] // c["block"]
    shape = (1, n_pages, c["page"], c["G"], c["d"])
    wide = 1 + 7 * (normal(c["G"], c["d"]) > 1.8)
    for name in ("k", "v"):
        x = normal(*shape[1:]) * (wide if name == "k" else 1) * torch.exp(0.5 * normal(n_pages, 1, c["G"], 1))
        x = x.view(n_pages, bpp, c["block"], c["G"], c["d"])
        scale = _scales_of(x.abs().amax((2, 4)))
        st[name + "_pages"] = (x / scale[:, :, None, :, None]).to(E4M3).view(shape)
        st[name + "_scale"] = scale.view(1, n_pages, bpp, c["G"])


def prepare(case, seed):
    c = case
    gen = torch.Generator("cuda").manual_seed(1000003 * seed + 31)
    dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    st = dict(case=c)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    lens = _lengths(c)
    if c["kind"] == "window":
        keys = [n + c["ahead"] if n else 0 for n in lens]
        cu = _cu(keys)
        q, k, v = normal(sum(lens), c["H"], c["d"]), normal(sum(keys), c["G"], c["d"]), normal(sum(keys), c["G"], c["d"])
        # every query looks at its sequence's first key, as trained attention does
        u = normal(c["G"], c["d"])
        u /= u.norm(dim=-1, keepdim=True)
        k[[a for a, n in zip(cu, keys) if n]] = 4 * math.sqrt(c["d"]) * u
        q += 2 * u.repeat_interleave(c["H"] // c["G"], 0)
        return dict(st, q=q.to(dt), k=k.to(dt), v=v.to(dt), cu_q=_ints(_cu(lens)), cu_k=_ints(cu))

    page, new = c["page"], _new_tokens(c) if c["kind"] == "write8" else [0] * c["n_seq"]
    before = [n - m for n, m in zip(lens, new)]
    n_pages = sum(-(-n // page) for n in lens) + 5
    table = _table(c, before, n_pages)
    count = [0] * n_pages
    for row in table:
        for x in row:
            if x >= 0:
                count[x] = 1
    st.update(table=_ints(table), lens=_ints(before), count=_ints(count))
    if c["kind"] == "window_decode":
        shape = (1, n_pages, page, c["G"], c["d"])
        st["k_pages"], st["v_pages"] = normal(*shape).to(dt), normal(*shape).to(dt)
    else:
        _fill8(st, c, n_pages, normal)
    if c["kind"] != "write8":
        return dict(st, q=normal(c["n_seq"], c["H"], c["d"]).to(dt))
    st.update(new=_ints(new), cu_new=_ints(_cu(new)), cu_back=_ints(_cu(_read_back(c))), total=sum(_read_back(c)))
    for name in ("k_new", "v_new"):  # (sequences differ in size, so that some blocks' scales grow)
        size = torch.exp(normal(c["n_seq"], c["G"], 1)).repeat_interleave(st["new"].long(), 0, output_size=sum(new))
        st[name] = (normal(sum(new), c["G"], c["d"]) * size).to(dt)
    st["ledger"] = [st["table"], st["lens"], st["count"]]  # a pass changes the ledger, and starts from this one
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
    return {"window": _plain_window, "window_decode": _plain_decode, "write8": _plain_write8, "decode8": _plain_decode}[kind](st)


def _own(st, kind):
    from paper_2510_19875_b200 import stream as S

    c = st["case"]
    if kind == "window":
        return S.prompt_attention(st["q"], st["k"], st["v"], st["cu_q"], st["cu_k"], window=c["window"], sinks=c["sinks"], want_lse=True)
    if "cache" not in st:  # the handle that a program keeps with its cache
        ledger = st["table"], st["lens"], st["count"]
        if kind == "window_decode":
            st["cache"] = S.PagedCache(st["k_pages"], st["v_pages"], *ledger)
        else:
            dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
            st["cache"] = S.PagedCache8(st["k_pages"], st["v_pages"], st["k_scale"], st["v_scale"], *ledger, dtype=dt)
    cache = st["cache"]
    if kind != "write8":
        return S.decode_attention(st["q"], cache, window=c["window"], sinks=c["sinks"], want_lse=True)
    info = S.cache_reserve(cache, st["new"])
    S.cache_write(cache, st["k_new"], st["v_new"], st["cu_new"], info=info)
    k, v = S.cache_read(cache, st["cu_back"], st["total"])
    return info, *st["ledger"], cache.k_scale, cache.v_scale, k, v


def _softmax_product(scores, v, how):
    """exp(scores) v over the last axis, divided by its sum; rows without a finite score give zeros and -inf."""
    top = scores.amax(-1, keepdim=True)
    shift = torch.where(top > -math.inf, top, 0.0)
    weights = torch.exp(scores - shift)
    total = weights.sum(-1)
    out = torch.einsum(how, weights, v) / torch.where(total > 0, total, 1.0).unsqueeze(-1)
    return out, shift.squeeze(-1) + torch.log(total)


def _plain_window(st):
    """All sequences at once, padded to the longest, some queries of it at a time with the keys that one of them sees."""
    c, q, k, v, cu_q, cu_k = (st[n] for n in ("case", "q", "k", "v", "cu_q", "cu_k"))
    H, G, d, n, window, sinks = c["H"], c["G"], c["d"], c["n_seq"], c["window"], c["sinks"]
    lens_q, lens_k = cu_q.diff(), cu_k.diff()
    N, M = q.shape[0], k.shape[0]
    out, lse = torch.empty(N + 1, H, d, device="cuda"), torch.empty(H, N + 1, device="cuda")
    at_once = max(1, min(c["longest"], 2 ** 30 // (n * H * min(c["longest"] + c["ahead"], window + sinks + 1024)), 1024))
    for a in range(0, c["longest"], at_once):
        i = torch.arange(a, min(a + at_once, c["longest"]), device="cuda")
        low = max(0, a + c["ahead"] - window + 1)  # (the last query sees its last key: as many keys in front of all queries)
        j = torch.arange(low, i.numel() + a + c["ahead"], device="cuda")
        if low > 0 and sinks > 0:
            j = torch.cat([torch.arange(min(sinks, low), device="cuda"), j])
        place = torch.where(i < lens_q[:, None], cu_q[:-1, None] + i, N)  # (what pads goes behind the end)
        there = j < lens_k[:, None]
        pos = i + c["ahead"]
        seen = (j <= pos[:, None]) & ((j > pos[:, None] - window) | (j < sinks))
        rows, keys = place.clamp(max=N - 1), (cu_k[:-1, None] + j).clamp(max=M - 1)
        qs = q[rows].float().view(n, i.numel(), G, H // G, d)
        ks, vs = k[keys].float(), v[keys].float()
        scores = torch.einsum("sighd,sjgd->sghij", qs, ks) / math.sqrt(d)
        scores.masked_fill_(~(seen[None] & there[:, None])[:, None, None], -math.inf)
        o, ls = _softmax_product(scores, vs, "sghij,sjgd->sghid")
        out[place.view(-1)] = o.permute(0, 3, 1, 2, 4).reshape(-1, H, d)
        lse[:, place.view(-1)] = ls.permute(1, 2, 0, 3).reshape(H, -1)
    return out[:N].to(q.dtype), lse[:, :N].contiguous()


def _values(st, pages, name):
    """What the whole pages [..] of a layer hold, [.., page, G, d] in fp32."""
    x = st[name + "_pages"][0]
    if x.dtype is not E4M3:
        return x[pages].float()
    scale = st[name + "_scale"][0][pages].repeat_interleave(st["case"]["block"], -2)
    return x.view(torch.uint8)[pages].view(E4M3).float() * scale.unsqueeze(-1)


def _plain_decode(st):
    c, q, table, lens = (st[n] for n in ("case", "q", "table", "lens"))
    n, width = table.shape
    tokens = width * c["page"]
    k, v = (_values(st, table.clamp(min=0), x).view(n, tokens, c["G"], c["d"]) for x in ("k", "v"))
    j = torch.arange(tokens, device="cuda")
    there = j < lens[:, None]
    if c["window"]:
        there = there & ((j >= lens[:, None] - c["window"]) | (j < c["sinks"]))
    v = torch.where(there[:, :, None, None], v, 0.0)
    scores = torch.einsum("sghd,sjgd->sghj", q.float().view(n, c["G"], -1, c["d"]), k) / math.sqrt(c["d"])
    scores.masked_fill_(~there[:, None, None], -math.inf)
    out, lse = _softmax_product(scores, v, "sghj,sjgd->sghd")
    return out.reshape(q.shape).to(q.dtype), lse.reshape(n, c["H"])


def _plain_write8(st):
    c, (table, lens, count), new, cu = st["case"], st["ledger"], st["new"], st["cu_new"]
    page, block, (n_slots, width), G = c["page"], c["block"], table.shape, c["G"]
    # room: the lowest free pages, all of it or none
    free = count == 0
    at = torch.arange(count.numel(), device="cuda")
    order, n_free = torch.sort(torch.where(free, at, at + count.numel())).values % count.numel(), free.sum()
    have, after = -(-lens // page), -(-(lens + new) // page)
    bad = ((new < 0) | (after > width)).sum()
    need = after - have
    total = need.sum()
    done = (bad == 0) & (total <= n_free)
    j = torch.arange(width, device="cuda")
    fresh = done & (j >= have[:, None]) & (j < after[:, None])
    which = (need.cumsum(0) - need)[:, None] + j - have[:, None]
    table.copy_(torch.where(fresh, order[which.clamp(0, order.numel() - 1)], table))
    taken = torch.where(done, total, 0)
    count.copy_(torch.where(free & (free.cumsum(0) <= taken), 1, count))
    lens.copy_(torch.where(done, lens + new, lens))
    info = torch.stack([done, total, n_free - taken, bad]).to(torch.int32)
    # whose block a new token is in, and the tokens that each slot's first block of them had before
    token = torch.arange(st["k_new"].shape[0], device="cuda", dtype=torch.int32)
    slot = torch.searchsorted(cu, token, right=True) - 1
    pos = lens[slot] - new[slot] + token - cu[slot]
    bpp = page // block
    in_page, in_block = (table[slot, pos // page] * page + pos % page).long(), (table[slot, pos // page] * bpp + pos % page // block).long()
    start = lens - new
    old = start // block * block + torch.arange(block, device="cuda")[:, None]  # [block, n_slots]
    is_old = (old < start) & (new > 0)
    old_page = table.gather(1, (old // page).clamp(max=width - 1).T.long()).T
    old_at, old_block = (torch.where(is_old, x, 0).long() for x in (old_page * page + old % page, old_page * bpp + old % page // block))
    partly = torch.zeros(count.numel() * bpp, dtype=torch.int32, device="cuda").index_add_(0, old_block.view(-1), is_old.view(-1).int()) > 0
    touched = torch.zeros_like(partly).index_fill_(0, in_block, True)
    for name in ("k", "v"):
        x, scale = st[name + "_new"].float(), st[name + "_scale"].view(-1, G)
        raw = st[name + "_pages"].view(torch.uint8).view(-1, G, c["d"])
        top = torch.zeros_like(scale).index_reduce_(0, in_block, x.abs().amax(-1), "amax")
        grown = torch.where(touched[:, None], torch.maximum(_scales_of(top), torch.where(partly[:, None], scale, 0.0)), scale)
        before = raw[old_at].view(E4M3).float() * (scale / grown)[old_block].unsqueeze(-1)
        kept = torch.where(is_old[..., None, None], before.to(E4M3).view(torch.uint8), raw[in_page[:1]])
        raw[torch.where(is_old, old_at, in_page[:1])] = kept  # (what is none of them goes to a place that is written next)
        raw[in_page] = (x / grown[in_block].unsqueeze(-1)).to(E4M3).view(torch.uint8)
        scale.copy_(grown)
    # the sequences' last tokens one behind the other
    cu_back = st["cu_back"]
    token = torch.arange(st["total"], device="cuda", dtype=torch.int32)
    slot = torch.searchsorted(cu_back, token, right=True) - 1
    pos = lens[slot] - (cu_back[slot + 1] - cu_back[slot]) + token - cu_back[slot]
    p, r = table[slot, pos // page].long(), (pos % page).long()
    values = []
    for name in ("k", "v"):
        raw, scale = st[name + "_pages"].view(torch.uint8)[0], st[name + "_scale"][0]
        values.append((raw[p, r].view(E4M3).float() * scale[p, r // block].unsqueeze(-1)).to(st["k_new"].dtype))
    return info, table, lens, count, st["k_scale"], st["v_scale"], *values


# ------------------------------------------------------------------------------------------------
def _seen(c, n):
    """Tokens of n that the last one sees."""
    return n if not c["window"] else min(n, c["window"]) + max(0, min(c["sinks"], n - c["window"]))


def work(case):
    c = case
    e = 4 if c["dtype"] == "f32" else 2
    lens, d, G = _lengths(c), c["d"], c["G"]
    if c["kind"] == "window":
        first, w, sinks = c["ahead"], c["window"], c["sinks"]

        def upto(x, most):  # the sum of min(p, most) over p = 1 .. x
            return 0 if x <= 0 else x * (x + 1) // 2 if x <= most else most * (most + 1) // 2 + (x - most) * most

        pairs = keys = 0
        for n in lens:
            if n:  # a query with p keys up to its own sees min(p, w) of them, and of those in front the sinks
                m = n + first
                pairs += upto(m, w) - upto(first, w) + upto(m - w, sinks) - upto(first - w, sinks)
                keys += m - max(0, first + 1 - w - sinks)
        q = sum(lens)
        return {"bytes": 2.0 * e * d * (q * c["H"] + keys * G) + 4.0 * q * c["H"], "flops": 4.0 * d * c["H"] * pairs}
    page = c["page"]
    if c["kind"] == "write8":  # the new tokens read and rounded, all of them read back and written out; the ledger as it is now
        back = _read_back(c)
        new, n, blocks = sum(_new_tokens(c)), sum(back), sum(-(-x // c["block"]) for x in back)
        n_pages = sum(-(-x // page) for x in lens) + 5
        return {"bytes": 2.0 * G * d * (e * new + n + e * n) + 8.0 * G * blocks + 4.0 * (n_pages + 4 * c["n_seq"]), "flops": 0.0}
    seen = [_seen(c, n) for n in lens]
    held = 1 if c["kind"] == "decode8" else e
    scales = 8.0 * G * sum(-(-n // c["block"]) for n in seen) if c["kind"] == "decode8" else 0.0
    ledger = 4.0 * (len(lens) + sum(-(-n // page) for n in seen))
    return {"bytes": 2.0 * d * (held * sum(seen) * G + e * len(lens) * c["H"]) + 4.0 * len(lens) * c["H"] + scales + ledger,
            "flops": 4.0 * d * c["H"] * sum(seen)}


def _exact_attention(q, k, v, first, window, sinks):
    """q [n, H, d], k and v [m, G, d] in 64 bits, query i is at position first + i of the keys; window 0: no end to what it sees.
    Some rows at a time, with the keys from the first that one of them sees, and the sinks in front of those."""
    n, H, d = q.shape
    m, G = k.shape[:2]
    out, lse = torch.zeros(n, H, d, dtype=torch.float64, device="cuda"), torch.full((H, n), -math.inf, dtype=torch.float64, device="cuda")
    if m == 0 or n == 0:
        return out, lse
    for a in range(0, n, 2048):
        b = min(n, a + 2048)
        row = torch.arange(first + a, first + b, device="cuda")[:, None]
        start = max(0, first + a - window + 1) if window else 0
        cols = list(range(min(sinks, start))) + list(range(start, min(m, first + b)))
        col = torch.tensor(cols, device="cuda")
        hidden = col > row
        if window:
            hidden |= (row - col >= window) & (col >= sinks)
        for h in range(H):
            s = (q[a:b, h].double() @ k[col, h * G // H].double().T) * d ** -0.5
            s.masked_fill_(hidden, -math.inf)
            lse[h, a:b] = torch.logsumexp(s, 1)
            out[a:b, h] = torch.softmax(s, 1) @ v[col, h * G // H].double()
    return out, lse


def exact(case, seed):
    c = case
    st = prepare(case, seed)
    if c["kind"] == "window":
        parts = []
        for s in range(c["n_seq"]):
            a, b, x, y = (int(t) for t in (st["cu_q"][s], st["cu_q"][s + 1], st["cu_k"][s], st["cu_k"][s + 1]))
            parts.append(_exact_attention(st["q"][a:b], st["k"][x:y], st["v"][x:y], (y - x) - (b - a), c["window"], c["sinks"]))
        return torch.cat([o for o, _ in parts]), torch.cat([x for _, x in parts], 1)
    page, lens = c["page"], _lengths(c)

    def tokens(name, table, s, n):
        """The first n tokens of sequence s in 64 bits."""
        pages = torch.tensor(table[s][: -(-n // page)], dtype=torch.int64, device="cuda")
        x = st[name + "_pages"][0].view(torch.uint8)[pages].view(st[name + "_pages"].dtype).double().view(-1, c["G"], c["d"])[:n]
        if c["kind"] != "window_decode":
            block_of = torch.arange(n, device="cuda") // c["block"]
            x = x * st[name + "_scale"][0][pages].double().view(-1, c["G"])[block_of].unsqueeze(-1)
        return x

    table = st["table"].tolist()
    if c["kind"] != "write8":
        parts = []
        for s, n in enumerate(lens):
            parts.append(_exact_attention(st["q"][s:s + 1], tokens("k", table, s, n), tokens("v", table, s, n), n - 1, c["window"], c["sinks"]))
        return torch.cat([o for o, _ in parts]), torch.cat([x.T for _, x in parts])
    # write8, sequence by sequence and block by block
    new, back, n_pages, block = _new_tokens(c), _read_back(c), st["count"].numel(), c["block"]
    before, count = st["lens"].tolist(), st["count"].tolist()
    heap, taken = [p for p in range(n_pages) if count[p] == 0], 0
    for s, n in enumerate(lens):
        for x in range(-(-before[s] // page), -(-n // page)):
            table[s][x] = heap.pop(0)
            count[table[s][x]] = 1
            taken += 1
    at = st["cu_new"].tolist()
    scales, values = [], []
    for name in ("k", "v"):
        scale, all_of_it = st[name + "_scale"].clone(), []
        for s, n in enumerate(lens):
            old = tokens(name, table, s, before[s])
            x = torch.cat([old, st[name + "_new"][at[s]:at[s + 1]].double()])
            size = torch.ones(n, c["G"], 1, dtype=torch.float64, device="cuda")
            # the scale of a block: by the largest of its new tokens, no smaller than the one it has
            first = before[s] // block
            n_blocks = -(-n // block)
            for b in range(n_blocks):
                p, r = table[s][b * block // page], b * block % page // block
                lo, hi = b * block, min(n, (b + 1) * block)
                if b >= first and new[s] > 0:
                    top = x[max(lo, before[s]):hi].abs().amax((0, 2))
                    e = torch.ceil(torch.log2(torch.clamp(top, min=1e-300) / 448.0))
                    e = e + (top > 448.0 * _two_to(e)).double() - (top <= 448.0 * _two_to(e - 1)).double()
                    mine = _two_to(e.clamp(-90, 120))
                    if lo < before[s]:
                        mine = torch.maximum(mine, scale[0, p, r].double())
                    scale[0, p, r] = mine.float()
                size[lo:hi] = scale[0, p, r].double()[None, :, None]
            y = x[first * block:] / size[first * block:]
            # the nearest number with four significant bits, of 2^-9 at least in the last place; ties to even
            unit = _two_to(torch.frexp(y.abs().clamp(min=2.0 ** -6)).exponent - 4)
            x = torch.cat([x[:first * block], torch.round(y / unit) * unit * size[first * block:]])
            all_of_it.append(x[n - back[s]:])
        scales.append(scale)
        values.append(torch.cat(all_of_it))
    return _ints([1, taken, len(heap), 0]), _ints(table), _ints(lens), _ints(count), *scales, *values
