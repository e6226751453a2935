"""The paged cache: its ledger against plain Python, the copies, and decode attention against 64 bits."""
import random
from types import SimpleNamespace

import pytest
import torch

from serve_helpers import Ledger, attention64, check, filled_cache, ints, offsets
from test_gpu_parity import S  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


# ------------------------------------------------------------------------------------------------
# Decode attention
# ------------------------------------------------------------------------------------------------
def decode_checked(S, q, cache, rows, layer=0, **kw):
    out, lse = S.decode_attention(q, cache, layer=layer, want_lse=True, **kw)
    torch.cuda.synchronize()
    for s, (k, v) in enumerate(rows):
        w = attention64(q[s:s + 1], k[layer], v[layer], None, kw.get("scale"))
        check(out[s:s + 1], lse[s:s + 1].T, w, k.shape[1], q.shape[2], q.dtype, s)
    return out, lse


@pytest.mark.parametrize("H,G", [(1, 1), (8, 2), (28, 4), (12, 12), (17, 1), (40, 2)])
@pytest.mark.parametrize("d,dtype", [(128, BF16), (64, BF16), (256, BF16), (32, BF16), (16, BF16), (64, F32), (128, F32), (256, F32), (32, F32), (16, F32)])
def test_decode(S, H, G, d, dtype):
    lens = [1, 0, 63, 64, 65, 500, 2, 1030]
    for page in (16, 1, 7, 64, 100):
        cache, rows, _ = filled_cache(S, lens, page, G, d, dtype, seed=page)
        q = torch.randn(len(lens), H, d, device="cuda").to(dtype)
        decode_checked(S, q, cache, rows)


@pytest.mark.parametrize("d,dtype", [(128, BF16), (64, F32), (32, BF16)])
@pytest.mark.parametrize("lens", [[20000], [1] * 700, [9000, 1, 0, 30], [0], [0, 0, 0]])
def test_decode_lengths(S, lens, d, dtype):
    """One long slot on every SM, more slots than units of a CTA, empty ones alone."""
    cache, rows, _ = filled_cache(S, lens, 32, 2, d, dtype)
    q = torch.randn(len(lens), 8, d, device="cuda").to(dtype)
    decode_checked(S, q, cache, rows)


@pytest.mark.parametrize("d,dtype", [(128, BF16), (64, F32)])
def test_decode_layers_layouts_and_scale(S, d, dtype):
    lens = [300, 17, 64, 0]
    for order in ("lpthd", "lphtd", "plthd", "hlptd", "pthld"):
        cache, rows, _ = filled_cache(S, lens, 16, 4, d, dtype, n_layers=3, order=order)
        q = torch.randn(len(lens), 2 * 8, d, device="cuda").to(dtype)
        for layer in (0, 2):
            decode_checked(S, q, cache, rows, layer=layer, scale=0.2)
    wide = torch.randn(len(lens), 20, d + 3, device="cuda").to(dtype)[:, 2:18, 3:]  # (q in an unaligned part of something wider)
    decode_checked(S, wide, cache, rows, layer=1)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_decode_of_rows_that_are_not_aligned(S, dtype):
    lens, d = [130, 40], 64
    cache, rows, led = filled_cache(S, lens, 16, 2, d, dtype)
    k, v = (torch.zeros(*x.shape[:4], d + 1, dtype=dtype, device="cuda")[..., 1:] for x in (cache.k, cache.v))
    k.copy_(cache.k), v.copy_(cache.v)
    q = torch.randn(2, 4, d, device="cuda").to(dtype)
    decode_checked(S, q, S.PagedCache(k, v, *led.tensors()), rows)


def test_decode_with_logits_that_outgrow_their_reference(S):
    lens = [900, 70]
    cache, rows, _ = filled_cache(S, lens, 16, 1, 128, BF16, garbage=0.0)
    for j, x in enumerate(cache.page_table[0].tolist()):
        if x >= 0:
            cache.k[:, x] *= j / 4
    rows[0][0][:] *= (torch.arange(900, device="cuda") // 16 / 4)[None, :, None, None].bfloat16()
    decode_checked(S, torch.randn(2, 8, 128, device="cuda").bfloat16(), cache, rows)


@pytest.mark.parametrize("d,dtype", [(128, BF16), (32, F32)])
def test_pages_outside_the_cache_are_left_out_and_recorded(S, d, dtype):
    lens = [200, 64, 90]
    cache, rows, _ = filled_cache(S, lens, 16, 2, d, dtype)
    q = torch.randn(3, 4, d, device="cuda").to(dtype)
    ws = torch.empty(S.stream_decode_workspace_bytes(cache.struct, 4), dtype=torch.uint8, device="cuda")
    decode_checked(S, q, cache, rows, workspace=ws)
    assert S.stream_read_stats(ws).error == 0
    cache.page_table[0, 3] = cache.n_pages
    cache.page_table[2, 0] = -1
    rows[0] = tuple(torch.cat([x[:, :48], x[:, 64:]], 1) for x in rows[0])
    rows[2] = tuple(x[:, 16:] for x in rows[2])
    decode_checked(S, q, cache, rows, workspace=ws)
    with pytest.raises(S.StreamError) as e:
        S.stream_read_stats(ws)
    assert e.value.status == S.STREAM_ERR_DEVICE_CHECK
    cache.page_table[1] = -5
    rows[1] = tuple(x[:, :0] for x in rows[1])
    decode_checked(S, q, cache, rows)
    cache.seq_len.copy_(ints([-3, 0, 2 ** 31 - 1]))  # none, none, and more than the table has room for
    rows[0] = tuple(x[:, :0] for x in rows[0])
    cache.page_table[2, 6:] = -1
    cache.k[:, cache.page_table[2, 5]] = 0  # (of the last page ten rows were written)
    cache.v[:, cache.page_table[2, 5]] = 0
    rows[2] = tuple(torch.cat([x[:, :64], torch.zeros_like(x[:, :16])], 1) for x in rows[2])
    decode_checked(S, q, cache, rows)


@pytest.mark.parametrize("d,dtype", [(128, BF16), (64, F32)])
def test_decode_again_on_streams_and_in_a_graph(S, d, dtype):
    lens = [700, 33, 0, 150]
    cache, rows, _ = filled_cache(S, lens, 16, 2, d, dtype)
    q = torch.randn(4, 8, d, device="cuda").to(dtype)
    a, la = S.decode_attention(q, cache, want_lse=True)
    torch.cuda.synchronize()
    sides = [torch.cuda.Stream() for _ in range(3)]
    got = [S.decode_attention(q, cache, want_lse=True, stream=s) for s in sides]
    torch.cuda.synchronize()
    for o, lse in got:
        assert torch.equal(o, a) and torch.equal(lse, la)
    n = S.stream_decode_workspace_bytes(cache.struct, 8)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")  # (one workspace for two graphs, replayed in turn)
    graphs = []
    for _ in range(2):
        x, o = q.clone(), torch.empty_like(q)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            S.decode_attention(x, cache, out=o, workspace=ws)
            S.decode_attention(o, cache, out=x, workspace=ws)
        graphs.append((g, x, o))
    for g, x, o in graphs * 2:
        for length in (lens, [0, 5, 20, 150], [1, 33, 0, 100]):
            cache.seq_len.copy_(ints(length))
            x.copy_(q)
            g.replay()
            e = S.decode_attention(q, cache)
            f = S.decode_attention(e, cache)
            torch.cuda.synchronize()
            assert torch.equal(o, e) and torch.equal(x, f)


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (F32, 64)])
def test_pages_beyond_32_bits(S, dtype, d):
    """A cache of more than 2^32 elements: decode, writes and copies on its last pages."""
    page, G = 64, 4
    n_pages = 2 ** 32 // (page * G * d) + 40
    k, v = (torch.empty(1, n_pages, page, G, d, dtype=dtype, device="cuda") for _ in range(2))
    led = Ledger(2, n_pages, page, 8)
    count = torch.ones(n_pages, dtype=torch.int32, device="cuda")
    count[-20:] = 0
    cache = S.PagedCache(k, v, ints(led.table), ints(led.len), count)
    new = [300, 70]
    info = S.cache_reserve(cache, ints(new))
    assert info.tolist() == [1, 7, 13, 0]
    assert cache.page_table[0, :5].tolist() == list(range(n_pages - 20, n_pages - 15))
    kk, vv = (torch.randn(370, G, d, device="cuda").to(dtype) for _ in range(2))
    S.cache_write(cache, kk, vv, ints([0, 300, 370]))
    rows = [(kk[None, :300], vv[None, :300]), (kk[None, 300:], vv[None, 300:])]
    q = torch.randn(2, 8, d, device="cuda").to(dtype)
    decode_checked(S, q, cache, rows)
    cache.ref_count[:50] = 0
    moves = S.cache_compact(cache)
    S.cache_copy_pages(cache, moves)
    assert moves.info.tolist() == [1, 50, 63, 0] and cache.page_table[0, 0] == 43  # (behind 43 pages that are in use, too)
    decode_checked(S, q, cache, rows)


# ------------------------------------------------------------------------------------------------
# The ledger
# ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("n_slots,n_pages,page,max_pages,steps", [(4, 20, 4, 8, 60), (33, 300, 16, 40, 40), (200, 5000, 2, 120, 12), (7, 3, 1, 3, 40), (1, 1, 3, 1, 12)])
def test_ledger_against_plain_python(S, n_slots, n_pages, page, max_pages, steps):
    """Random calls, refused ones among them; small ledgers by one CTA, large ones by eight."""
    rng = random.Random(n_slots)
    cache = S.new_cache(n_slots, n_pages, page, max_pages, 1, 16, dtype=F32)
    led = Ledger(n_slots, n_pages, page, max_pages)
    seen = set()
    for step in range(steps):
        what = rng.choice(["reserve", "reserve", "fork", "free", "compact"])
        if what == "reserve":
            most = rng.choice([0, 1, page, 3 * page, max_pages * page])
            new = [rng.randint(0, most) if rng.random() < 0.4 else 0 for _ in range(n_slots)]
            if rng.random() < 0.15:
                new[rng.randrange(n_slots)] = rng.choice([-1, -2 ** 31, 2 ** 31 - 1])
            info, want = S.cache_reserve(cache, ints(new)), led.reserve(new)
        elif what == "fork":
            empty = [s for s in range(n_slots) if led.len[s] == 0]
            full = [s for s in range(n_slots) if led.len[s] > 0] or [0]
            parent = [-1] * n_slots
            for s in empty:
                if rng.random() < 0.5:
                    parent[s] = rng.choice(full)
            if rng.random() < 0.2:
                parent[rng.randrange(n_slots)] = rng.choice([0, n_slots, n_slots - 1, 2 ** 31 - 1])
            moves, (pairs, want) = S.cache_fork(cache, ints(parent)), led.fork(parent)
            assert moves.pairs.tolist() == pairs
            info = moves.info
        elif what == "free":
            done = [rng.choice([0, 0, 1, -1, 5]) for _ in range(n_slots)]
            info, want = S.cache_free(cache, ints(done)), led.free(done)
        else:
            moves, (pairs, want) = S.cache_compact(cache), led.compact()
            assert moves.pairs.tolist() == pairs
            info = moves.info
        assert info.tolist() == want, (step, what)
        assert led.same(cache), (step, what)
        seen.add((what, want[0]))
    if n_slots > 1:
        assert {("reserve", 0), ("reserve", 1), ("fork", 1), ("free", 1), ("compact", 1)} <= seen


@pytest.mark.parametrize("n_pages", [50, 40000])
def test_entries_that_cannot_be_are_passed_over(S, n_pages):
    """A table that names pages outside the cache, counts and lengths that cannot be: nothing outside is touched, and it is said."""
    cache = S.new_cache(4, n_pages, 4, 6, 1, 16, dtype=F32)
    assert S.cache_reserve(cache, ints([20, 8, 0, 4])).tolist() == [1, 8, n_pages - 8, 0]
    cache.page_table[0, 1] = n_pages
    cache.page_table[0, 2] = -7
    cache.ref_count[cache.page_table[1, 0]] = 0
    cache.seq_len[3] = 2 ** 30
    info = S.cache_free(cache, ints([1, 1, 0, 1])).tolist()
    assert info[0] == 1 and info[3] >= 4
    assert (cache.page_table == -1).all() and (cache.seq_len == 0).all() and (cache.ref_count >= 0).all()
    cache.seq_len.copy_(ints([-1, 25, 0, 0]))
    for parent in ([-1, -1, 0, -1], [-1, -1, 1, -1]):
        moves = S.cache_fork(cache, ints(parent))
        assert moves.info.tolist()[0] == 0 and moves.info.tolist()[3] == 1 and (moves.pairs == -1).all()
    assert S.cache_reserve(cache, ints([1, 0, 0, 0])).tolist()[3] == 2


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("order", ["lpthd", "lphtd", "plthd", "hlptd"])
def test_copies_of_pages(S, order, dtype):
    for page, G, d, pad in ((16, 4, 64, 0), (5, 3, 16, 0), (7, 1, 128, 1), (1, 2, 32, 0), (64, 8, 128, 0)):
        L, n_pages = 3, 11
        sizes = dict(l=L, p=n_pages, t=page, h=G, d=d + pad)
        perm = [order.index(x) for x in "lpthd"]
        k, v = (torch.randn([sizes[x] for x in order], device="cuda").to(dtype).permute(perm)[..., pad:] for _ in range(2))
        cache = S.PagedCache(k, v, ints([[-1]]), ints([0]), torch.zeros(n_pages, dtype=torch.int32, device="cuda"))
        pairs = [[0, 5], [3, 10], [n_pages, 1], [2, -1], [-1, -1], [0, 7], [4, 6], [8, 9]]
        info = ints([1, 7, 0, 0])  # (the last pair is behind the count)
        want_k, want_v = k.clone(), v.clone()
        for a, b in ((0, 5), (3, 10), (0, 7), (4, 6)):
            want_k[:, b], want_v[:, b] = k[:, a], v[:, a]
        S.cache_copy_pages(cache, S.CacheMoves(ints(pairs), info))
        assert torch.equal(cache.k, want_k) and torch.equal(cache.v, want_v)
        for n in (0, -4):
            S.cache_copy_pages(cache, S.CacheMoves(ints([[1, 2]]), ints([1, n, 0, 0])))
        assert torch.equal(cache.k, want_k)
        S.cache_copy_pages(cache, S.CacheMoves(ints([[1, 2]]), ints([1, 2 ** 31 - 1, 0, 0])))  # (no more than there are)
        assert torch.equal(cache.k[:, 2], want_k[:, 1])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("page,G,d,order,pad", [(16, 4, 64, "lpthd", 0), (5, 3, 16, "lphtd", 0), (7, 2, 128, "hlptd", 1), (64, 8, 128, "plthd", 0)])
def test_writes_of_new_tokens(S, page, G, d, order, pad, dtype):
    lens, new = [3, 0, 40, 1, 0, 90, 64], [5, 0, 77, 1, 200, 0, 1]
    cache, rows, led = filled_cache(S, lens, page, G, d, dtype, n_layers=2, spare=-(-sum(new) // page) + len(new), order=order, max_pages=-(-300 // page))
    want = led.reserve(new)
    assert S.cache_reserve(cache, ints(new)).tolist() == want and want[0] == 1 and led.same(cache)
    cu = offsets(new)
    k, v = (torch.randn(cu[-1] + 9, G + 1, d + pad, device="cuda").to(dtype)[:, 1:, pad:] for _ in range(2))
    before_k, before_v = cache.k.clone(), cache.v.clone()
    S.cache_write(cache, k, v, ints(cu), layer=1)
    for s, n in enumerate(new):
        for i in range(n):
            pos = lens[s] + i
            x, t = led.table[s][pos // page], pos % page
            before_k[1, x, t], before_v[1, x, t] = k[cu[s] + i], v[cu[s] + i]
    assert torch.equal(cache.k.view(torch.int16 if dtype is BF16 else torch.int32), before_k.view(torch.int16 if dtype is BF16 else torch.int32))
    assert torch.equal(cache.v.view(torch.int16 if dtype is BF16 else torch.int32), before_v.view(torch.int16 if dtype is BF16 else torch.int32))


def test_writes_that_cannot_be_are_passed_over(S):
    cache = S.new_cache(3, 6, 4, 2, 1, 16, dtype=F32)
    assert S.cache_reserve(cache, ints([8, 3, 0])).tolist() == [1, 3, 3, 0]
    cache.k.zero_(), cache.v.zero_()
    cache.page_table[0, 1] = 6
    k = torch.ones(12, 1, 16, device="cuda")
    S.cache_write(cache, k, k, ints([0, 9, 12, 12]))  # slot 0 has one row more than tokens
    S.cache_write(cache, k, k, ints([-5, -5, -5, 2 ** 31 - 1]))  # an empty slot with rows
    S.cache_write(cache, k, k, ints([12, 4, 0, 0]))
    assert cache.k.sum() == 16 * (4 + 3) and cache.k[0, 3:].sum() == 0
    S.cache_write(cache, k[:0], k[:0], ints([0, 0, 0, 0]))


@pytest.mark.parametrize("n_slots", [3, 40])
def test_nothing_is_written_after_a_refused_reserve(S, n_slots):
    cache = S.new_cache(n_slots, 4, 4, 400, 2, 16, dtype=F32)  # (by one CTA, by eight)
    cache.k.zero_(), cache.v.zero_()
    cu = ints([0] + [8] * n_slots)
    k = torch.ones(8, 2, 16, device="cuda")
    for new, done in ((8, 1), (16, 0), (8, 1)):
        info = S.cache_reserve(cache, ints([new] + [0] * (n_slots - 1)))
        before = cache.k.clone(), cache.v.clone()
        S.cache_write(cache, k * new, k * new, cu, info=info)
        assert info[0] == done
        if not done:
            assert torch.equal(cache.k, before[0]) and torch.equal(cache.v, before[1])
    assert cache.seq_len[0] == 16 and cache.k.min() == 8


def test_many_slots(S):
    n = 3000
    cache = S.new_cache(n, 2 * n, 8, 4, 1, 16, dtype=F32)
    led = Ledger(n, 2 * n, 8, 4)
    new = [i % 13 for i in range(n)]
    assert S.cache_reserve(cache, ints(new)).tolist() == led.reserve(new) and led.same(cache)
    cu = offsets(new)
    k, v = torch.randn(cu[-1], 1, 16, device="cuda"), torch.randn(cu[-1], 1, 16, device="cuda")
    S.cache_write(cache, k, v, ints(cu))
    q = torch.randn(n, 2, 16, device="cuda")
    out, lse = S.decode_attention(q, cache, want_lse=True)
    for s in list(range(0, n, 271)) + [n - 1]:
        w = attention64(q[s:s + 1], k[cu[s]:cu[s + 1]], v[cu[s]:cu[s + 1]], None)
        check(out[s:s + 1], lse[s:s + 1].T, w, 13, 16, F32, s)


# ------------------------------------------------------------------------------------------------
# All of them together
# ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("d,dtype,page", [(128, BF16, 16), (64, BF16, 5), (64, F32, 8)])
def test_chains_forked_from_prompts(S, d, dtype, page):
    """Prompts into the cache, chains forked from them, tokens one by one, ends and a compaction on the way: every token's attention
    is that of a prompt of all the chain's tokens."""
    H, G, n_slots, layers = 8, 2, 9, 2
    rng = random.Random(d)
    cache = S.new_cache(n_slots, 120, page, 40, G, d, n_layers=layers, dtype=dtype)
    cache.k.fill_(float("nan")), cache.v.fill_(float("nan"))
    text = [None] * n_slots  # the keys and values of every slot's tokens: [layers, n, G, d]

    def grow(new):
        assert S.cache_reserve(cache, ints(new)).tolist()[0] == 1
        cu = offsets(new)
        fresh = [tuple(torch.randn(cu[-1], G, d, device="cuda").to(dtype) for _ in range(2)) for _ in range(layers)]
        for layer, (k, v) in enumerate(fresh):
            S.cache_write(cache, k, v, ints(cu), layer=layer)
        for s, n in enumerate(new):
            if n:
                part = tuple(torch.stack([x[i][cu[s]:cu[s + 1]] for x in fresh]) for i in range(2))
                text[s] = part if text[s] is None else tuple(torch.cat(p, 1) for p in zip(text[s], part))
        return cu

    def look(cu):
        q = torch.randn(n_slots, H, d, device="cuda").to(dtype)
        nothing = torch.zeros(layers, 0, G, d, dtype=dtype, device="cuda")
        rows = [t if t is not None else (nothing, nothing) for t in text]
        for layer in range(layers):
            out, lse = decode_checked(S, q, cache, rows, layer=layer)
            alive = [s for s in range(n_slots) if text[s] is not None]
            cu_k = offsets([rows[s][0].shape[1] for s in alive])
            whole, whole_lse = S.prompt_attention(q[alive].contiguous(), torch.cat([rows[s][0][layer] for s in alive]),
                                                  torch.cat([rows[s][1][layer] for s in alive]), ints(list(range(len(alive) + 1))),
                                                  ints(cu_k), want_lse=True)
            for i, s in enumerate(alive):
                w = attention64(q[s:s + 1], rows[s][0][layer], rows[s][1][layer], None)
                check(whole[i:i + 1], whole_lse[:, i:i + 1], w, cu_k[i + 1] - cu_k[i], d, dtype)

    look(grow([33, 0, 0, 2 * page, 0, 0, 1, 0, 0]))
    parent = [-1, 0, 0, -1, 3, -1, -1, 6, -1]
    moves = S.cache_fork(cache, ints(parent))
    assert moves.info.tolist()[:2] == [1, sum(text[p][0].shape[1] % page != 0 for p in parent if p >= 0)]
    S.cache_copy_pages(cache, moves)
    for s, p in enumerate(parent):
        if p >= 0:
            text[s] = tuple(x.clone() for x in text[p])
    look(None)
    for _ in range(3):
        look(grow([rng.randint(0, 2) if text[s] is not None else 0 for s in range(n_slots)]))
    done = [1, 0, 0, 0, 1, 0, 0, 0, 0]
    assert S.cache_free(cache, ints(done)).tolist()[0] == 1
    for s, x in enumerate(done):
        if x:
            text[s] = None
    look(None)
    moves = S.cache_compact(cache)
    S.cache_copy_pages(cache, moves)
    used = cache.n_pages - moves.info.tolist()[2]
    assert (cache.ref_count[:used] > 0).all() and (cache.ref_count[used:] == 0).all()
    look(None)
    look(grow([5 if text[s] is not None else 0 for s in range(n_slots)]))


def test_a_step_captured_in_a_graph(S):
    """Room, writes and attention of one new token, captured once and replayed: the cache grows with every replay."""
    n, G, H, d, page = 5, 2, 8, 128, 16
    cache = S.new_cache(n, 60, page, 10, G, d)
    grown = S.new_cache(n, 60, page, 10, G, d)
    one, cu = ints([1] * n), ints(list(range(n + 1)))
    k, v = (torch.zeros(n, G, d, dtype=BF16, device="cuda") for _ in range(2))
    q = torch.zeros(n, H, d, dtype=BF16, device="cuda")
    ws = torch.empty(S.stream_decode_workspace_bytes(cache.struct, H), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        info = S.cache_reserve(cache, one)
        S.cache_write(cache, k, v, cu)
        out = S.decode_attention(q, cache, workspace=ws)
    cache.page_table.fill_(-1), cache.seq_len.zero_(), cache.ref_count.zero_()
    for step in range(40):
        for x in (k, v, q):
            x.copy_(torch.randn_like(x))
        graph.replay()
        assert info.tolist()[0] == 1
        S.cache_reserve(grown, one)
        S.cache_write(grown, k, v, cu)
        assert torch.equal(out, S.decode_attention(q, grown))
    assert cache.seq_len.tolist() == [40] * n and torch.equal(cache.page_table, grown.page_table)


@pytest.mark.parametrize("handle", [False, True])
@pytest.mark.parametrize("what", ["prompt", "decode", "reserve", "fork", "free", "compact"])
def test_memory_of_a_call_on_another_stream(S, what, handle):
    """What a call on another stream writes to (results, a workspace) is not handed to the current one while the call has yet to run."""
    q, k = torch.randn(4, 8, 64, device="cuda").to(BF16), torch.randn(4, 2, 64, device="cuda").to(BF16)
    cu, ones, parent = ints([0, 4]), ints([0, 1, 0, 0]), ints([-1, 0, -1, -1])
    side = torch.cuda.Stream()
    for waiting in (False, True):  # (the first time kernels are loaded, which waits for the GPU)
        cache, _, _ = filled_cache(S, [70, 0, 33, 0], 16, 2, 64, BF16)
        calls = dict(prompt=lambda: S.prompt_attention(q, k, k, cu, want_lse=True, stream=st), decode=lambda: S.decode_attention(q, cache, want_lse=True, stream=st),
                     reserve=lambda: S.cache_reserve(cache, ones, stream=st), fork=lambda: S.cache_fork(cache, parent, stream=st),
                     free=lambda: S.cache_free(cache, ones, stream=st), compact=lambda: S.cache_compact(cache, stream=st))
        sizes = [16, 32, 2 * 4 * 8 * 64, 4 * 4 * 8, 8 * (cache.n_pages // 2), S.stream_decode_workspace_bytes(cache.struct, 8)]
        st = side.cuda_stream if handle else side
        torch.cuda.synchronize()
        if waiting:
            with torch.cuda.stream(side):
                torch.cuda._sleep(400_000_000)  # (a fifth of a second)
        calls[what]()
        here = [torch.full((n,), 77, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(4)]
        torch.cuda.current_stream().synchronize()
        assert not (waiting and side.query())
        side.synchronize()
        for x in here:
            assert (x == 77).all()


LEDGER_CALLS = dict(reserve=lambda S, c, x, **kw: S.cache_reserve(c, x, **kw), fork=lambda S, c, x, **kw: S.cache_fork(c, x, **kw),
                    free=lambda S, c, x, **kw: S.cache_free(c, x, **kw), compact=lambda S, c, x, **kw: S.cache_compact(c, **kw))


def own_arrays(S, lens):
    """The arrays of a cache, to be held without a handle."""
    cache, _, led = filled_cache(S, lens, 16, 2, 64, BF16, spare=40, max_pages=12)
    return (cache.k, cache.v, cache.page_table, cache.seq_len, cache.ref_count), led


@pytest.mark.parametrize("how", ["stream", "handle", "current"])
@pytest.mark.parametrize("what", LEDGER_CALLS)
def test_a_ledger_call_hands_out_memory_of_its_own_stream(S, monkeypatch, what, how):
    """The workspace of a call on another stream is that stream's memory, so that one who lets go of the handle at once gets none of
    it on the current one. Nothing is launched here: the calls are recorded."""
    arrays, _ = own_arrays(S, [70, 0, 33, 0])
    x = ints([0, 1, 0, 0] if what != "fork" else [-1, 0, -1, -1])
    side = torch.cuda.Stream()
    cache = S.PagedCache(*arrays)
    n = S.stream_cache_workspace_bytes(cache.struct)
    seen = []
    with monkeypatch.context() as m:
        m.setattr(S, "_lib", SimpleNamespace(**{f"stream_cache_{w}": lambda *a: seen.append(a) or 0 for w in LEDGER_CALLS}))
        if how == "current":
            with torch.cuda.stream(side):
                LEDGER_CALLS[what](S, cache, x)
        else:
            LEDGER_CALLS[what](S, cache, x, stream=side if how == "stream" else side.cuda_stream)
        del cache
    (args,) = seen
    at, size, stream = args[-3:]
    assert size >= n and at % 256 == 0 and stream == side.cuda_stream
    here = [torch.empty(m, dtype=torch.uint8, device="cuda") for m in (n, 512, 1024, 2048) for _ in range(8)]
    assert all(y.data_ptr() + y.numel() <= at or at + size <= y.data_ptr() for y in here)


@pytest.mark.parametrize("how", ["stream", "current", "graph"])
@pytest.mark.parametrize("what", LEDGER_CALLS)
def test_the_handle_is_let_go_before_its_call_has_run(S, what, how):
    """The ledger's arrays held by the program, a handle made for one call only, and the current stream busy with memory of its own."""
    lens = [70, 0, 33, 0, 90, 16]
    x = dict(reserve=[20, 17, 0, 100, 3, 1], fork=[-1, 0, -1, 2, -1, -1], free=[1, 0, 0, 0, 1, 0], compact=None)[what]
    dev = None if x is None else ints(x)
    side = torch.cuda.Stream()
    for waiting in (False, True):  # (the first time kernels are loaded, which waits for the GPU)
        arrays, led = own_arrays(S, lens)
        if what == "compact":
            S.cache_free(S.PagedCache(*arrays), ints([0, 0, 1, 0, 0, 0])), led.free([0, 0, 1, 0, 0, 0])
        torch.cuda.synchronize()
        if how == "graph":
            graph, cache = torch.cuda.CUDAGraph(), S.PagedCache(*arrays)
            with torch.cuda.graph(graph):
                got = LEDGER_CALLS[what](S, cache, dev)
            del cache
        with torch.cuda.stream(side):
            if waiting:
                torch.cuda._sleep(200_000_000)
            if how == "graph":
                graph.replay()
            elif how == "current":
                got = LEDGER_CALLS[what](S, S.PagedCache(*arrays), dev)
        if how == "stream":
            got = LEDGER_CALLS[what](S, S.PagedCache(*arrays), dev, stream=side)
        here = [torch.full((m,), 0x77, dtype=torch.uint8, device="cuda") for m in (512, 1024, 2048) for _ in range(8)]
        torch.cuda.current_stream().synchronize()
        side.synchronize()
        assert all((y == 0x77).all() for y in here)
        if what in ("fork", "compact"):
            pairs, want = led.fork(x) if what == "fork" else led.compact()
            assert got.info.tolist() == want and got.pairs.tolist() == pairs
        else:
            assert got.tolist() == (led.reserve(x) if what == "reserve" else led.free(x))
        assert led.same(SimpleNamespace(page_table=arrays[2], seq_len=arrays[3], ref_count=arrays[4], device=arrays[0].device))
