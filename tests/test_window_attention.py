"""Attention with a sliding window and sinks against 64 bits: of packed prompts and over a paged cache, every kernel and its edges."""
import pytest
import torch

from serve8_helpers import masked64, seen_by
from serve_helpers import check, filled_cache, ints, offsets
from test_dense_attention import inputs
from test_gpu_parity import S  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def want(q, k, v, cu_q, cu_k, window, sinks, scale=None):
    parts = []
    for a, b, x, y in zip(cu_q, cu_q[1:], cu_k, cu_k[1:]):
        parts.append(masked64(q[a:b], k[x:y], v[x:y], seen_by(b - a, y - x, window, sinks), scale))
    return tuple(torch.cat([p[i] for p in parts], 1 if i == 1 else 0) for i in range(4))


def run(S, q, k, v, cu_q, cu_k, window, sinks, **kw):
    n, H, d = cu_q[-1], q.shape[1], q.shape[2]
    out = torch.full((q.shape[0], H, d), 7.0, dtype=q.dtype, device="cuda")
    lse = torch.full((H, q.shape[0]), 7.0, device="cuda")
    S.prompt_attention(q, k, v, ints(cu_q), ints(cu_k), window=window, sinks=sinks, out=out, lse_out=lse, **kw)
    torch.cuda.synchronize()
    S.stream_check_device_status()
    assert (out[n:] == 7).all() and (lse[:, n:] == 7).all()  # rows of no sequence
    check(out[:n], lse[:, :n], want(q, k, v, cu_q, cu_k, window, sinks, kw.get("scale")), max([b - a for a, b in zip(cu_k, cu_k[1:])]), d, q.dtype,
          (window, sinks))
    return out, lse


FORMS = [(8, 2, 128, BF16), (7, 1, 64, BF16), (28, 4, 128, BF16), (16, 16, 128, BF16), (33, 1, 64, BF16), (1, 1, 128, BF16), (8, 2, 256, BF16), (6, 2, 32, BF16),
         (7, 1, 16, BF16), (300, 2, 64, BF16), (1, 1, 64, F32), (8, 2, 128, F32), (6, 2, 32, F32), (3, 1, 16, F32), (2, 1, 256, F32)]
LENS = [([1], [1]), ([128, 129], [128, 129]), ([5, 0, 700, 1], [5, 0, 700, 1]), ([3, 300], [600, 301]),
        ([200, 7, 150], [60, 0, 149])]   # (the last: queries that see nothing, no keys at all)


@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("H,G,d,dtype", FORMS)
def test_window(S, H, G, d, dtype, lens):
    q, k, v, cu_q, cu_k = inputs(H, G, d, *lens, dtype, behind=5, seed=H + d)
    for window, sinks in ((1, 0), (1, 1), (5, 3), (64, 0), (100, 130), (129, 4), (300, 1), (700, 0), (2 ** 31 - 1, 2 ** 31 - 1)):
        run(S, q, k, v, cu_q, cu_k, window, sinks)


@pytest.mark.parametrize("H,G,d,n,dtype", [(8, 2, 128, 3001, BF16), (4, 4, 64, 2500, BF16), (2, 1, 64, 2500, F32), (2, 2, 128, 1999, F32), (4, 1, 256, 1500, BF16),
                                           (2, 1, 256, 1500, F32)])
def test_long_sequences(S, H, G, d, n, dtype):
    q, k, v, cu_q, cu_k = inputs(H, G, d, [n, 77], [n, 500], dtype, seed=n)
    for window, sinks in ((37, 4), (512, 0), (1000, 200)):
        run(S, q, k, v, cu_q, cu_k, window, sinks)


@pytest.mark.parametrize("H,G,d,lens", [(28, 4, 128, [700, 1500, 0, 333, 64, 2000, 1, 129]), (128, 1, 64, [5000, 300]), (4, 2, 64, [i % 23 for i in range(1300)])])
def test_more_items_than_ctas(S, H, G, d, lens):
    q, k, v, cu_q, cu_k = inputs(H, G, d, lens, lens, BF16, behind=7, seed=H)
    run(S, q, k, v, cu_q, cu_k, 200, 3)


@pytest.mark.parametrize("d,dtype", [(128, BF16), (64, BF16), (256, BF16), (64, F32), (256, F32)])
def test_a_window_as_long_as_the_sequences_is_the_dense_call(S, d, dtype):
    q, k, v, cu_q, cu_k = inputs(4, 2, d, [300, 40], [300, 70], dtype)
    dense = S.prompt_attention(q, k, v, ints(cu_q), ints(cu_k), want_lse=True)
    for window, sinks in ((300, 0), (1, 300), (2 ** 31 - 1, 0)):
        out, lse = S.prompt_attention(q, k, v, ints(cu_q), ints(cu_k), window=window, sinks=sinks, want_lse=True)
        assert torch.equal(out, dense[0]) and torch.equal(lse, dense[1])


@pytest.mark.parametrize("d,dtype", [(128, BF16), (64, BF16), (32, BF16), (64, F32), (256, F32)])
def test_logits_that_outgrow_their_reference_and_late_first_keys(S, d, dtype):
    q, k, v, cu_q, cu_k = inputs(4, 2, d, [700], [700], dtype, sink=False)
    k *= (torch.arange(700, device="cuda")[:, None, None] / 60).to(dtype)
    run(S, q, k, v, cu_q, cu_k, 150, 2)
    run(S, q, k.flip(0).contiguous(), v, cu_q, cu_k, 150, 2, scale=0.3)


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 64)])
def test_strides(S, dtype, d):
    q, k, v, cu_q, cu_k = inputs(8, 2, d, [150, 290], [150, 290], dtype)
    a = run(S, q, k, v, cu_q, cu_k, 60, 5)
    b = run(S, *(x.transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v)), cu_q, cu_k, 60, 5)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    odd = torch.zeros(440, 12, d + 1, dtype=dtype, device="cuda")
    odd[:, :8, 1:], odd[:, 8:10, 1:], odd[:, 10:, 1:] = q, k, v
    run(S, odd[:, :8, 1:], odd[:, 8:10, 1:], odd[:, 10:, 1:], cu_q, cu_k, 60, 5)


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 32), (F32, 64), (F32, 256)])
def test_offsets_that_cannot_be_stay_inside(S, dtype, d):
    q, k, v, cu_q, cu_k = inputs(4, 2, d, [200], [200], dtype)
    out, lse = S.prompt_attention(q, k, v, ints([-50, 2 ** 31 - 1]), ints([-2 ** 31, 900]), window=50, sinks=2, want_lse=True)
    check(out, lse, want(q, k, v, [0, 200], [0, 200], 50, 2), 200, d, dtype)
    cu = ints([0, 200] * 150)  # sequences that overlap since the offsets fall: twice the same rows
    out, lse = S.prompt_attention(q, k, v, cu, window=50, sinks=2, want_lse=True)
    torch.cuda.synchronize()
    S.stream_check_device_status()
    check(out, lse, want(q, k, v, [0, 200], [0, 200], 50, 2), 200, d, dtype)


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 256), (F32, 64)])
def test_on_streams_and_in_a_graph(S, dtype, d):
    q, k, v, cu_q, cu_k = inputs(8, 2, d, [300, 0, 45], [300, 0, 45], dtype)
    cu = ints(cu_q)
    a, la = S.prompt_attention(q, k, v, cu, window=70, sinks=3, want_lse=True)
    torch.cuda.synchronize()
    outs = [S.prompt_attention(q, k, v, cu, window=70, sinks=3, want_lse=True, stream=st) for st in [torch.cuda.Stream() for _ in range(3)]]
    torch.cuda.synchronize()
    assert all(torch.equal(o, a) and torch.equal(lse, la) for o, lse in outs)
    lens = cu.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, lse = S.prompt_attention(q, k, v, lens, window=70, sinks=3, want_lse=True)
        o2 = S.prompt_attention(o, k, v, lens, window=9)
    for other in ([0, 1, 200, 345], [0, 300, 300, 345]):
        lens.copy_(ints(other))
        graph.replay()
        torch.cuda.synchronize()
        e, le = S.prompt_attention(q, k, v, ints(other), window=70, sinks=3, want_lse=True)
        assert torch.equal(o, e) and torch.equal(lse, le) and torch.equal(o2, S.prompt_attention(e, k, v, ints(other), window=9))


@pytest.mark.parametrize("n", [200_000])
def test_a_long_prompt(S, n):
    m, d = 77, 128
    q, k, v = (torch.randn(n + m, h, d, device="cuda", dtype=BF16) for h in (8, 4, 4))
    out, lse = S.prompt_attention(q, k, v, ints([0, n, n + m]), window=1500, sinks=5, want_lse=True)
    torch.cuda.synchronize()
    S.stream_check_device_status()
    check(out[n:], lse[:, n:], masked64(q[n:], k[n:], v[n:], seen_by(m, m, 1500, 5)), m, d, BF16)
    for at in (0, 1000, n // 2 + 1, n - 3):
        lo = max(0, at - 1600)
        keys = torch.cat([torch.arange(min(5, lo), device="cuda"), torch.arange(lo, at + 3, device="cuda")])
        p = torch.arange(at, at + 3, device="cuda")[:, None]
        seen = (keys <= p) & ((keys > p - 1500) | (keys < 5))
        check(out[at:at + 3], lse[:, at:at + 3], masked64(q[at:at + 3], k[keys], v[keys], seen), len(keys), d, BF16)


# ------------------------------------------------------------------------------------------------
# One new token over a paged cache
# ------------------------------------------------------------------------------------------------
def decode_checked(S, q, cache, rows, window, sinks, layer=0, **kw):
    out, lse = S.decode_attention(q, cache, layer=layer, window=window, sinks=sinks, want_lse=True, **kw)
    torch.cuda.synchronize()
    for s, (k, v) in enumerate(rows):
        m = k.shape[1]
        w = masked64(q[s:s + 1], k[layer], v[layer], seen_by(1, m, window, sinks)[:, :m] if m else None, kw.get("scale"))
        check(out[s:s + 1], lse[s:s + 1].T, w, m, q.shape[2], q.dtype, (s, window, sinks))
    return out, lse


WINDOWS = [(1, 0), (1, 1), (40, 0), (64, 65), (100, 4), (513, 200), (2 ** 31 - 1, 0)]


@pytest.mark.parametrize("H,G", [(1, 1), (8, 2), (28, 4), (17, 1), (40, 2)])
@pytest.mark.parametrize("d,dtype", [(128, BF16), (64, BF16), (256, BF16), (32, BF16), (16, BF16), (64, F32), (128, F32), (256, F32), (32, F32), (16, F32)])
def test_decode(S, H, G, d, dtype):
    lens = [1, 0, 63, 64, 65, 500, 2, 1030]
    for i, page in enumerate((16, 1, 7, 64, 100)):
        cache, rows, _ = filled_cache(S, lens, page, G, d, dtype, seed=page)
        q = torch.randn(len(lens), H, d, device="cuda").to(dtype)
        for window, sinks in WINDOWS[i:i + 3]:
            decode_checked(S, q, cache, rows, window, sinks)


@pytest.mark.parametrize("d,dtype", [(128, BF16), (64, F32)])
@pytest.mark.parametrize("lens", [[20000], [1] * 700, [9000, 1, 0, 30], [0]])
def test_decode_lengths(S, lens, d, dtype):
    cache, rows, _ = filled_cache(S, lens, 32, 2, d, dtype)
    q = torch.randn(len(lens), 8, d, device="cuda").to(dtype)
    for window, sinks in ((1000, 4), (8000, 100)):
        decode_checked(S, q, cache, rows, window, sinks)


@pytest.mark.parametrize("d,dtype,off", [(128, BF16, 0), (64, F32, 0), (64, BF16, 1), (64, F32, 1)])
@pytest.mark.parametrize("page", [16, 5])
def test_decode_reads_nothing_between_the_sinks_and_the_window(S, d, dtype, off, page):
    """Keys that are not seen may be anything, their pages' entries too, and are not recorded; off: rows that are not aligned."""
    lens, window, sinks = [300, 17, 200, 0], 33, 6
    cache, rows, led = filled_cache(S, lens, page, 2, d, dtype, n_layers=2)
    if off:
        k, v = (torch.zeros(*x.shape[:4], d + 1, dtype=dtype, device="cuda")[..., 1:] for x in (cache.k, cache.v))
        k.copy_(cache.k), v.copy_(cache.v)
        cache = S.PagedCache(k, v, *led.tensors())
    q = torch.randn(4, 8, d, device="cuda").to(dtype)
    ws = torch.empty(S.stream_decode_workspace_bytes(cache.struct, 8), dtype=torch.uint8, device="cuda")
    a = decode_checked(S, q, cache, rows, window, sinks, layer=1, workspace=ws, scale=0.2)
    for s, n in enumerate(lens):
        for j in range(sinks, n - window):
            x = led.table[s][j // page]
            cache.k[:, x, j % page] = float("nan")
            cache.v[:, x, j % page] = float("inf")
        for j in range(-(-n // page)):
            if j * page >= sinks and (j + 1) * page <= n - window:
                cache.page_table[s, j] = -7 if j % 2 else cache.n_pages
    b = S.decode_attention(q, cache, layer=1, window=window, sinks=sinks, want_lse=True, workspace=ws, scale=0.2)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert S.stream_read_stats(ws).error == 0
    cache.page_table[0, (300 - 10) // page] = -1  # one that is seen
    S.decode_attention(q, cache, layer=1, window=window, sinks=sinks, workspace=ws)
    with pytest.raises(S.StreamError):
        S.stream_read_stats(ws)


@pytest.mark.parametrize("d,dtype", [(128, BF16), (64, F32)])
def test_decode_layouts(S, d, dtype):
    lens = [300, 17, 64, 0]
    for order in ("lphtd", "plthd", "hlptd"):
        cache, rows, _ = filled_cache(S, lens, 16, 4, d, dtype, n_layers=3, order=order)
        q = torch.randn(len(lens), 20, d + 3, device="cuda").to(dtype)[:, 2:18, 3:]
        decode_checked(S, q, cache, rows, 50, 3, layer=2)


@pytest.mark.parametrize("d,dtype", [(128, BF16), (64, F32)])
def test_decode_on_streams_and_in_a_graph(S, d, dtype):
    lens = [700, 33, 0, 150]
    cache, rows, _ = filled_cache(S, lens, 16, 2, d, dtype)
    q = torch.randn(4, 8, d, device="cuda").to(dtype)
    a, la = S.decode_attention(q, cache, window=90, sinks=2, want_lse=True)
    torch.cuda.synchronize()
    got = [S.decode_attention(q, cache, window=90, sinks=2, want_lse=True, stream=s) for s in [torch.cuda.Stream() for _ in range(3)]]
    torch.cuda.synchronize()
    assert all(torch.equal(o, a) and torch.equal(lse, la) for o, lse in got)
    ws = torch.full((S.stream_decode_workspace_bytes(cache.struct, 8),), 255, dtype=torch.uint8, device="cuda")
    graphs = []
    for _ in range(2):  # (one workspace for two graphs, replayed in turn)
        x, o = q.clone(), torch.empty_like(q)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            S.decode_attention(x, cache, window=90, sinks=2, out=o, workspace=ws)
            S.decode_attention(o, cache, out=x, workspace=ws)
        graphs.append((g, x, o))
    for g, x, o in graphs * 2:
        for length in (lens, [0, 5, 20, 150], [1, 33, 0, 100]):
            cache.seq_len.copy_(ints(length))
            x.copy_(q)
            g.replay()
            e = S.decode_attention(q, cache, window=90, sinks=2)
            f = S.decode_attention(e, cache)
            torch.cuda.synchronize()
            assert torch.equal(o, e) and torch.equal(x, f)


@pytest.mark.parametrize("d,dtype", [(128, BF16), (64, F32), (256, F32)])
def test_decode_under_a_window_as_long_as_the_slots_is_the_dense_call(S, d, dtype):
    cache, rows, _ = filled_cache(S, [700, 33, 0, 150], 16, 2, d, dtype)
    q = torch.randn(4, 8, d, device="cuda").to(dtype)
    a = S.decode_attention(q, cache, want_lse=True)
    b = S.decode_attention(q, cache, window=700, want_lse=True)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# ------------------------------------------------------------------------------------------------
# Packed rows out of the pages
# ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("d,dtype,off", [(128, BF16, 0), (64, F32, 0), (32, BF16, 0), (16, F32, 0), (64, BF16, 1)])
def test_cache_read(S, d, dtype, off):
    lens = [300, 17, 64, 0, 1]
    for order, page in (("lpthd", 16), ("lphtd", 7), ("hlptd", 64)):
        cache, rows, led = filled_cache(S, lens, page, 3, d, dtype, n_layers=2, order=order)
        if off:
            k, v = (torch.zeros(*x.shape[:4], d + 1, dtype=dtype, device="cuda")[..., 1:] for x in (cache.k, cache.v))
            k.copy_(cache.k), v.copy_(cache.v)
            cache = S.PagedCache(k, v, *led.tensors())
        for take in (lens, [5, 17, 0, 0, 1]):
            cu = offsets(take)
            k, v = (torch.full((cu[-1] + 4, 3, d), 7.0, dtype=dtype, device="cuda") for _ in range(2))
            a = S.cache_read(cache, ints(cu), cu[-1] + 4, layer=1, out=(k, v))
            assert a[0] is k and a[1] is v
            for x, i in ((k, 0), (v, 1)):
                assert torch.equal(x[:cu[-1]], torch.cat([r[i][1, n - m:n] for r, n, m in zip(rows, lens, take)]))
                assert (x[cu[-1]:] == 7).all()  # rows of no slot
    # more rows than tokens, and a page that is none: zeros
    cache.page_table[1, 0] = -1
    k, v = S.cache_read(cache, ints([0, 0, 17, 85, 85, 85]), 85)
    assert not k[:17].any() and not k[17:21].any() and torch.equal(k[21:], rows[2][0][0]) and torch.equal(v[21:], rows[2][1][0])
    assert S.cache_read(cache, ints([0] * 6), 0)[0].shape == (0, 3, d)


def test_a_prompt_in_pieces(S):
    """Tokens written to the pages, read back, and attended to: as the whole prompt at once."""
    G, H, d, page, lens = 2, 8, 128, 16, [150, 40, 333]
    q, k, v, cu, _ = inputs(H, G, d, lens, lens, BF16)
    whole = S.prompt_attention(q, k, v, ints(cu), window=70, sinks=4)
    cache = S.new_cache(3, 60, page, 24, G, d)
    done = [0, 0, 0]
    got = torch.empty_like(whole)
    for step in ([100, 40, 1], [0, 0, 300], [50, 0, 32]):
        rows = torch.cat([torch.arange(a + b, a + b + n, device="cuda") for a, b, n in zip(cu, done, step)])
        info = S.cache_reserve(cache, ints(step))
        S.cache_write(cache, k[rows], v[rows], ints(offsets(step)), info=info)
        done = [a + n for a, n in zip(done, step)]
        kk, vv = S.cache_read(cache, ints(offsets(done)), sum(done))
        part = S.prompt_attention(q[rows], kk, vv, ints(offsets(step)), ints(offsets(done)), window=70, sinks=4)
        got[rows] = part
    w = want(q, k, v, cu, cu, 70, 4)
    check(got, None, w, 333, d, BF16)
    check(whole, None, w, 333, d, BF16)
