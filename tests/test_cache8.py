"""The paged cache in 8 bits: what is written and read back against plain Python, and decode attention against 64 bits."""
import pytest
import torch

from serve8_helpers import E4M3, Slots8, check8, empty_cache8, filled_cache8, rounded8, scale_of, seen_by, masked64
from serve_helpers import check, ints, offsets
from test_gpu_parity import S  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


# ------------------------------------------------------------------------------------------------
# Writing and reading back
# ------------------------------------------------------------------------------------------------
def written(S, cache, held, steps, layer, gen, size, wide=False):
    """Step by step: new tokens for every slot, in the library and in plain Python."""
    G, d = cache.n_kv_heads, cache.d
    for i, new in enumerate(steps):
        rows = [(torch.randn(sum(new), G, d, generator=gen, device="cuda") * size(i)).to(cache.dtype) for _ in range(2)]
        info = S.cache_reserve(cache, ints(new))
        assert info.tolist()[0] == 1
        k, v = rows
        if wide:  # parts of wider rows, which are not aligned
            both = torch.zeros(sum(new), 2 * G, d + 1, dtype=cache.dtype, device="cuda")
            both[:, :G, 1:], both[:, G:, 1:] = k, v
            k, v = both[:, :G, 1:], both[:, G:, 1:]
        S.cache_write(cache, k, v, ints(offsets(new)), layer=layer, info=info)
        at = offsets(new)
        for s in range(len(new)):
            for kv in range(2):
                held.write(s, layer, kv, rows[kv][at[s]:at[s + 1]])


def compare(S, cache, held, layer):
    """All tokens read back, the scales, and whether what belongs to nobody is as it was."""
    lens = cache.seq_len.tolist()
    cu = offsets(lens)
    back = S.cache_read(cache, ints(cu), cu[-1], layer=layer)
    table, page, block = cache.page_table.tolist(), cache.page_size, cache.block
    for kv, (pages, scale) in enumerate(((cache.k, cache.k_scale), (cache.v, cache.v_scale))):
        nobody, unscaled = torch.ones(pages.shape[1:3], dtype=torch.bool, device="cuda"), torch.ones(scale.shape[1:3], dtype=torch.bool, device="cuda")
        for s, n in enumerate(lens):
            x, z = held.held[s][layer][kv]
            assert x.shape[0] == n
            assert torch.equal(back[kv][cu[s]:cu[s + 1]].double(), x.to(cache.dtype).double()), (s, kv)
            for b in range(-(-n // block)):
                p, r = table[s][b * block // page], b * block % page // block
                assert torch.equal(scale[layer, p, r].double(), z[b]), (s, kv, b)
                unscaled[p, r] = False
            for j in range(n):
                nobody[table[s][j // page], j % page] = False
        assert (pages.view(torch.uint8)[layer][nobody] == 127).all()
        assert torch.isnan(scale[layer][unscaled]).all()


@pytest.mark.parametrize("d,dtype", [(128, BF16), (64, F32), (32, BF16), (16, F32), (256, BF16), (256, F32)])
@pytest.mark.parametrize("page,block", [(16, 16), (64, 16), (24, 8), (7, 7), (5, 1), (128, 128), (64, 64)])
def test_written_and_read_back(S, d, dtype, page, block):
    """Blocks that begin, go on and are finished; values that grow, so that scales do, and shrink."""
    steps = [[0, 5, 33, 1, 130], [1, 1, 1, 1, 1], [40, 0, 2, 1, 100], [1, 1, 0, 1, 1], [3, 3, 3, 3, 3]]
    lens = [sum(x) for x in zip(*steps)]
    need = sum(-(-n // page) for n in lens)
    gen = torch.Generator("cuda").manual_seed(d + page)
    cache, _ = empty_cache8(S, 5, page, block, 3, d, dtype, need, n_layers=2, max_pages=max(-(-n // page) for n in lens) + 1)
    held = Slots8(5, 2, block, 3, d)
    written(S, cache, held, steps, 1, gen, lambda i: (1.0, 7.0, 0.1, 300.0, 2.0)[i])
    compare(S, cache, held, 1)
    assert (cache.k.view(torch.uint8)[0] == 127).all() and torch.isnan(cache.v_scale[0]).all()  # the other layer


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_layouts_and_rows_that_are_not_aligned(S, dtype):
    steps, page, block, G, d = [[20, 5, 70], [1, 1, 1], [30, 20, 9]], 32, 16, 2, 64
    for order, scale_order in (("lphtd", "lphb"), ("hlptd", "hbpl"), ("pltdh", "lpbh")):
        if order.endswith("h"):
            order = "plthd"
        gen = torch.Generator("cuda").manual_seed(1)
        cache, _ = empty_cache8(S, 3, page, block, G, d, dtype, 9, n_layers=2, order=order, scale_order=scale_order)
        held = Slots8(3, 2, block, G, d)
        written(S, cache, held, steps, 0, gen, lambda i: 1.0 + i)
        compare(S, cache, held, 0)
    gen = torch.Generator("cuda").manual_seed(1)
    cache, led = empty_cache8(S, 3, page, block, G, d, dtype, 9)
    k, v = (torch.full((*x.shape[:4], d + 1), 127, dtype=torch.uint8, device="cuda").view(E4M3)[..., 1:] for x in (cache.k, cache.v))
    cache = S.PagedCache8(k, v, cache.k_scale, cache.v_scale, *led.tensors(), dtype=dtype)
    held = Slots8(3, 1, block, G, d)
    written(S, cache, held, steps, 0, gen, lambda i: 1.0 + i, wide=True)
    compare(S, cache, held, 0)


def test_values_at_the_edges(S):
    """Zeros, scales at their limits, values on and next to a border, ties, infinities and NaN."""
    d, block = 16, 2
    up = lambda x: torch.nextafter(torch.tensor(x), torch.tensor(float("inf"))).item()  # noqa: E731
    rows = [[0.0, 0.0], [448.0, 1.0], [up(448.0), 1.0], [-448.0, 17.0], [2.0 ** 127 * 1.75, 1.0], [3.4028234663852886e38, -3e38], [2.0 ** -82 * 1.75, 0.0],
            [2.0 ** -90, 2.0 ** -99], [2.0 ** -149, 2.0 ** -120], [17.0, 18.0], [19.0, 21.0], [448.0, 2.0 ** -10], [448.0, 3 * 2.0 ** -10], [448.0, 2.0 ** -6 * 0.97]]
    x = torch.zeros(len(rows) * block, 1, d)
    for i, (a, b) in enumerate(rows):
        x[2 * i, 0, 3], x[2 * i + 1, 0, 7] = a, b
    x = x.cuda()
    cache, _ = empty_cache8(S, 1, 4, block, 1, d, F32, 7, max_pages=8)
    held = Slots8(1, 1, block, 1, d)
    info = S.cache_reserve(cache, ints([x.shape[0]]))
    S.cache_write(cache, x, -x, ints([0, x.shape[0]]), info=info)
    held.write(0, 0, 0, x), held.write(0, 0, 1, -x)
    compare(S, cache, held, 0)
    inf, nan = float("inf"), float("nan")
    y = torch.zeros(6, 1, d, device="cuda")
    y[0, 0, 0], y[1, 0, 1] = inf, -inf
    y[2, 0, 0], y[3, 0, 1] = nan, 3.0
    y[4, 0], y[5, 0] = nan, nan
    cache, _ = empty_cache8(S, 1, 4, block, 1, d, F32, 7, max_pages=8)
    info = S.cache_reserve(cache, ints([6]))
    S.cache_write(cache, y, y, ints([0, 6]), info=info)
    k, _ = S.cache_read(cache, ints([0, 6]), 6)
    assert k[0, 0, 0] == inf and k[1, 0, 1] == -inf and k[0, 0, 1] == 0  # (448 scales of 2^120 are more than fp32 holds)
    assert torch.isnan(k[2, 0, 0]) and k[3, 0, 1] == 3 and k[2, 0, 1] == 0
    assert torch.isnan(k[4:]).all() and (cache.k_scale[0, 1, 0] == 2.0 ** -90).all()


def test_more_elements_than_a_group_holds_and_many_slots(S):
    gen = torch.Generator("cuda").manual_seed(2)
    cache, _ = empty_cache8(S, 2, 256, 256, 1, 256, F32, 8)
    held = Slots8(2, 1, 256, 1, 256)
    written(S, cache, held, [[600, 3], [1, 500], [250, 1]], 0, gen, lambda i: 1.0 + 3 * i)
    compare(S, cache, held, 0)
    n = 1500
    cache, _ = empty_cache8(S, n, 16, 16, 1, 16, BF16, n, max_pages=2)
    held = Slots8(n, 1, 16, 1, 16)
    written(S, cache, held, [[i % 4 for i in range(n)], [(i + 1) % 2 for i in range(n)]], 0, gen, lambda i: 1.0 + i)
    compare(S, cache, held, 0)


def test_a_refused_reserve_and_what_cannot_be(S):
    gen = torch.Generator("cuda").manual_seed(3)
    cache, led = empty_cache8(S, 2, 16, 16, 2, 32, BF16, 2, spare=0)
    held = Slots8(2, 1, 16, 2, 32)
    written(S, cache, held, [[20, 0]], 0, gen, lambda i: 1.0)
    x = torch.randn(30, 2, 32, device="cuda").bfloat16()
    info = S.cache_reserve(cache, ints([10, 20]))  # a page too many
    assert info.tolist()[0] == 0
    S.cache_write(cache, x, x, ints([0, 10, 30]), info=info)
    compare(S, cache, held, 0)
    # rows of no slot; more rows than tokens: the last ones count; no page
    before = [t.clone() for t in (cache.k.view(torch.uint8), cache.k_scale)]
    S.cache_write(cache, x, x, ints([30, 30, 30]))
    S.cache_write(cache, x, x, ints([0, 0, 30]))   # slot 1 has no tokens
    assert torch.equal(before[0], cache.k.view(torch.uint8)) and torch.equal(before[1].nan_to_num(-1), cache.k_scale.nan_to_num(-1))
    S.cache_write(cache, x, x, ints([-5, 2 ** 31 - 1, 7]))  # clamped: all 30 rows are slot 0's, which has 20 tokens
    held.held[0][0] = [[torch.zeros(0, 2, 32, device="cuda", dtype=torch.float64), torch.zeros(0, 2, device="cuda", dtype=torch.float64)] for _ in range(2)]
    for kv in range(2):
        held.write(0, 0, kv, x[10:])
    compare(S, cache, held, 0)
    cache.page_table[0, 1] = 2 ** 30
    before = cache.k.clone().view(torch.uint8)
    S.cache_write(cache, x * 2, x * 2, ints([0, 4, 4]))  # (the last four lie on that page)
    k, _ = S.cache_read(cache, ints([0, 20, 20]), 20)
    assert torch.equal(before, cache.k.view(torch.uint8)) and not k[16:].any() and k[:16].any()


# ------------------------------------------------------------------------------------------------
# Decode attention
# ------------------------------------------------------------------------------------------------
def decode_checked(S, q, cache, held, window=0, sinks=0, layer=0, **kw):
    out, lse = S.decode_attention(q, cache, layer=layer, window=window, sinks=sinks, want_lse=True, **kw)
    torch.cuda.synchronize()
    for s in range(q.shape[0]):
        k, v = (held.held[s][layer][kv][0] for kv in range(2))
        z, m = held.scales_by_token(s, layer, 1), k.shape[0]
        if m:
            seen = seen_by(1, m, window, sinks)[0]
            k, v, z = k[seen], v[seen], z[seen]
        check8(out[s], lse[s], q[s], k, v, z, kw.get("scale"), q.dtype, (s, window, sinks))
    return out, lse


@pytest.mark.parametrize("H,G", [(1, 1), (8, 2), (28, 4), (12, 12), (17, 1), (40, 2)])
@pytest.mark.parametrize("d,dtype", [(128, BF16), (64, BF16), (256, BF16), (32, BF16), (16, BF16), (64, F32), (128, F32), (256, F32), (32, F32), (16, F32)])
def test_decode(S, H, G, d, dtype):
    lens = [1, 0, 63, 64, 65, 500, 2, 1030]
    for i, (page, block) in enumerate(((16, 16), (64, 32), (7, 7), (3, 1), (100, 20))):
        cache, held, _ = filled_cache8(S, lens, page, block, G, d, dtype, seed=page)
        q = torch.randn(len(lens), H, d, device="cuda").to(dtype)
        decode_checked(S, q, cache, held)
        decode_checked(S, q, cache, held, *((1, 0), (40, 3), (64, 65), (513, 200), (2 ** 31 - 1, 9))[i])


@pytest.mark.parametrize("d,dtype", [(128, BF16), (64, F32), (32, BF16)])
@pytest.mark.parametrize("lens", [[20000], [1] * 700, [9000, 1, 0, 30], [0], [0, 0, 0]])
def test_decode_lengths(S, lens, d, dtype):
    cache, held, _ = filled_cache8(S, lens, 32, 32, 2, d, dtype)
    q = torch.randn(len(lens), 8, d, device="cuda").to(dtype)
    decode_checked(S, q, cache, held)
    decode_checked(S, q, cache, held, 3000, 70)


@pytest.mark.parametrize("d,dtype", [(128, BF16), (64, F32), (256, BF16)])
def test_decode_with_sizes_far_apart(S, d, dtype):
    """Blocks of values and keys that differ by many powers of two: keys that outgrow the reference, values next to none."""
    lens = [900, 70]
    n = 60
    q = torch.randn(2, 8, d, device="cuda").to(dtype)
    for size in (torch.linspace(0, 6, n), torch.linspace(6, 0, n), 2.0 ** torch.linspace(-30, 3, n), 2.0 ** torch.linspace(3, -30, n),
                 torch.where(torch.arange(n) % 3 == 0, 0.0, 1.0)):
        cache, held, _ = filled_cache8(S, lens, 16, 16, 1, d, dtype, size=size.cuda())
        decode_checked(S, q, cache, held)
        decode_checked(S, q * 2.0 ** -40, cache, held, scale=2.0 ** 40)
    # values alone
    cache, held, _ = filled_cache8(S, lens, 16, 16, 1, d, dtype)
    f = 2.0 ** torch.randint(-50, 50, cache.v_scale.shape, device="cuda")
    cache.v_scale *= f
    for s, m in enumerate(lens):
        by_block = f[0][cache.page_table[s, :-(-m // 16)].long(), 0].double()
        x, z = held.held[s][0][1]
        held.held[s][0][1] = [x * by_block.repeat_interleave(16, 0)[:m, :, None], z * by_block]
    decode_checked(S, q, cache, held)


def test_decode_with_scales_that_are_no_powers_of_two(S):
    lens, d = [300, 41], 64
    for dtype in (BF16, F32):
        cache, held, _ = filled_cache8(S, lens, 16, 8, 2, d, dtype)
        for kv, scale in ((0, cache.k_scale), (1, cache.v_scale)):
            f = 1 + torch.rand(scale.shape, device="cuda")
            new = scale * f
            for s, m in enumerate(lens):
                old, by_block = (x[0][cache.page_table[s, :-(-m // 16)].long()].reshape(-1, 2)[:-(-m // 8)].double() for x in (scale, new))
                x, z = held.held[s][0][kv]
                held.held[s][0][kv] = [x * (by_block / old).repeat_interleave(8, 0)[:m, :, None], by_block]
            scale.copy_(new)
        decode_checked(S, torch.randn(2, 8, d, device="cuda").to(dtype), cache, held)


@pytest.mark.parametrize("d,dtype", [(128, BF16), (64, F32)])
def test_decode_layers_layouts_and_scale(S, d, dtype):
    lens = [300, 17, 64, 0]
    for order, scale_order in (("lpthd", "lpbh"), ("lphtd", "hlpb"), ("hlptd", "bplh")):
        cache, held, _ = filled_cache8(S, lens, 32, 16, 4, d, dtype, n_layers=3, order=order, scale_order=scale_order)
        q = torch.randn(len(lens), 20, d + 3, device="cuda").to(dtype)[:, 2:18, 3:]  # (an unaligned part of something wider)
        for layer in (0, 2):
            decode_checked(S, q, cache, held, layer=layer, scale=0.2)


@pytest.mark.parametrize("d,dtype", [(64, BF16), (32, F32), (256, BF16)])
def test_decode_of_rows_that_are_not_aligned(S, d, dtype):
    lens = [130, 40]
    cache, held, led = filled_cache8(S, lens, 16, 16, 2, d, dtype)
    k, v = (torch.zeros(*x.shape[:4], d + 1, dtype=torch.uint8, device="cuda")[..., 1:] for x in (cache.k, cache.v))
    k.copy_(cache.k.view(torch.uint8)), v.copy_(cache.v.view(torch.uint8))
    odd = S.PagedCache8(k.view(E4M3), v.view(E4M3), cache.k_scale, cache.v_scale, *led.tensors(), dtype=dtype)
    q = torch.randn(2, 4, d, device="cuda").to(dtype)
    a = decode_checked(S, q, odd, held, 50, 3)
    b = decode_checked(S, q, cache, held, 50, 3)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("d,dtype", [(128, BF16), (32, F32)])
def test_pages_outside_the_cache_and_what_is_not_seen(S, d, dtype):
    lens, window, sinks = [200, 64, 90], 33, 5
    cache, held, _ = filled_cache8(S, lens, 16, 16, 2, d, dtype)
    q = torch.randn(3, 4, d, device="cuda").to(dtype)
    ws = torch.empty(S.stream_decode_workspace_bytes(cache.struct, 4), dtype=torch.uint8, device="cuda")
    a = decode_checked(S, q, cache, held, window, sinks, workspace=ws)
    for s, n in enumerate(lens):
        for j in range(1, (n - window) // 16):
            x = int(cache.page_table[s, j])
            cache.k.view(torch.uint8)[:, x], cache.v.view(torch.uint8)[:, x], cache.k_scale[:, x], cache.v_scale[:, x] = 127, 127, float("nan"), float("nan")
            cache.page_table[s, j] = -1 if j % 2 else x
    b = S.decode_attention(q, cache, window=window, sinks=sinks, want_lse=True, workspace=ws)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and S.stream_read_stats(ws).error == 0
    cache, held, _ = filled_cache8(S, lens, 16, 16, 2, d, dtype)
    cache.page_table[0, 3] = cache.n_pages
    for kv in range(2):
        x, z = held.held[0][0][kv]
        held.held[0][0][kv] = [torch.cat([x[:48], x[64:]]), torch.cat([z[:3], z[4:]])]
    decode_checked(S, q, cache, held, workspace=ws)
    with pytest.raises(S.StreamError) as e:
        S.stream_read_stats(ws)
    assert e.value.status == S.STREAM_ERR_DEVICE_CHECK
    cache.seq_len.copy_(ints([-3, 0, 2 ** 31 - 1]))  # none, none, and more than the table has room for
    cache.page_table[2, 5:] = -1
    for kv in range(2):
        for s in (0, 1):
            held.held[s][0][kv] = [held.held[s][0][kv][0][:0], held.held[s][0][kv][1][:0]]
        x, z = held.held[2][0][kv]
        held.held[2][0][kv] = [x[:80], z[:5]]
    decode_checked(S, q, cache, held)


@pytest.mark.parametrize("d,dtype", [(128, BF16), (64, F32)])
def test_decode_again_on_streams_and_in_a_graph(S, d, dtype):
    lens = [700, 33, 0, 150]
    cache, held, _ = filled_cache8(S, lens, 16, 16, 2, d, dtype)
    q = torch.randn(4, 8, d, device="cuda").to(dtype)
    a, la = S.decode_attention(q, cache, want_lse=True)
    torch.cuda.synchronize()
    got = [S.decode_attention(q, cache, want_lse=True, stream=s) for s in [torch.cuda.Stream() for _ in range(3)]]
    torch.cuda.synchronize()
    assert all(torch.equal(o, a) and torch.equal(lse, la) for o, lse in got)
    ws = torch.full((S.stream_decode_workspace_bytes(cache.struct, 8),), 255, dtype=torch.uint8, device="cuda")
    graphs = []
    for _ in range(2):  # (one workspace for two graphs, replayed in turn)
        x, o = q.clone(), torch.empty_like(q)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            S.decode_attention(x, cache, out=o, workspace=ws)
            S.decode_attention(o, cache, window=20, sinks=2, out=x, workspace=ws)
        graphs.append((g, x, o))
    for g, x, o in graphs * 2:
        for length in (lens, [0, 5, 20, 150], [1, 33, 0, 100]):
            cache.seq_len.copy_(ints(length))
            x.copy_(q)
            g.replay()
            e = S.decode_attention(q, cache)
            f = S.decode_attention(e, cache, window=20, sinks=2)
            torch.cuda.synchronize()
            assert torch.equal(o, e) and torch.equal(x, f)


@pytest.mark.parametrize("d,dtype", [(128, BF16), (64, F32), (16, BF16)])
def test_outputs_that_lie_off_their_boundaries_and_very_long_windows(S, d, dtype):
    """Contiguous outputs one element behind a boundary; windows beyond 32 bits."""
    lens = [70, 0, 600]
    cache, held, _ = filled_cache8(S, lens, 16, 16, 2, d, dtype)
    q = torch.randn(3, 4, d, device="cuda").to(dtype)
    a, la = decode_checked(S, q, cache, held)
    odd = torch.zeros(q.numel() + 1, dtype=dtype, device="cuda")[1:].view(q.shape)
    lse = torch.zeros(3 * 4 + 1, device="cuda")[1:].view(3, 4)
    assert S.decode_attention(q, cache, out=odd, lse_out=lse)[0] is odd and torch.equal(odd, a) and torch.equal(lse, la)
    b, lb = S.decode_attention(q, cache, window=2 ** 40, sinks=2 ** 40, want_lse=True)
    assert torch.equal(a, b) and torch.equal(la, lb)
    cu = ints(offsets(lens))
    k, v = S.cache_read(cache, cu, 670)
    out = [torch.zeros(k.numel() + 1, dtype=dtype, device="cuda")[1:].view(k.shape) for _ in range(2)]
    S.cache_read(cache, cu, 670, out=out)
    assert torch.equal(out[0], k) and torch.equal(out[1], v)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_offsets_beyond_32_bits(S, dtype):
    """Pages further apart than 2^31 elements in all."""
    lens, d, page = [150, 37], 64, 16
    cache, held, led = filled_cache8(S, lens, page, 16, 2, d, dtype, spare=0)
    n = cache.n_pages
    k, v = (torch.zeros(n * 2 ** 28, dtype=torch.uint8, device="cuda").as_strided((1, n, page, 2, d), (0, 2 ** 28, 128, 64, 1)) for _ in range(2))
    k.copy_(cache.k.view(torch.uint8)), v.copy_(cache.v.view(torch.uint8))
    far = S.PagedCache8(k.view(E4M3), v.view(E4M3), cache.k_scale.clone(), cache.v_scale.clone(), *led.tensors(), dtype=dtype)
    q = torch.randn(2, 4, d, device="cuda").to(dtype)
    a, b = decode_checked(S, q, cache, held), decode_checked(S, q, far, held)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    cu = ints(offsets(lens))
    assert all(torch.equal(x, y) for x, y in zip(S.cache_read(cache, cu, 187), S.cache_read(far, cu, 187)))
    rows = torch.randn(2, 2, d, device="cuda").to(dtype) * 9
    for c in (cache, far):
        S.cache_write(c, rows, rows, ints([0, 1, 2]))
    assert all(torch.equal(x, y) for x, y in zip(S.cache_read(cache, cu, 187), S.cache_read(far, cu, 187)))


# ------------------------------------------------------------------------------------------------
# All of it together
# ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("d,dtype,odd", [(64, BF16, 0), (32, F32, 0), (32, BF16, 1)])
def test_chains_that_are_prompted_forked_continued_freed_and_compacted(S, d, dtype, odd):
    G, H, page, block, n_layers, n_slots = 2, 6, 16, 8, 2, 6
    if odd:  # pages whose bytes lie off every boundary
        led = empty_cache8(S, n_slots, page, block, G, d, dtype, 60, n_layers=n_layers, max_pages=12)[1]
        k, v = (torch.zeros(n_layers, 63, page, G, d + 1, dtype=torch.uint8, device="cuda").view(E4M3)[..., 1:] for _ in range(2))
        z = [torch.zeros(n_layers, 63, page // block, G, device="cuda") for _ in range(2)]
        cache = S.PagedCache8(k, v, *z, *led.tensors(), dtype=dtype)
    else:
        cache = S.new_cache8(n_slots, 63, page, 12, G, d, block=block, n_layers=n_layers, dtype=dtype)
    held = Slots8(n_slots, n_layers, block, G, d)
    gen = torch.Generator("cuda").manual_seed(4)

    def step(new):
        at = offsets(new)
        info = S.cache_reserve(cache, ints(new))
        assert info.tolist()[0] == 1
        for layer in range(n_layers):
            rows = [(torch.randn(at[-1], G, d, generator=gen, device="cuda") * (1 + layer)).to(dtype) for _ in range(2)]
            S.cache_write(cache, *rows, ints(at), layer=layer, info=info)
            for s in range(n_slots):
                for kv in range(2):
                    held.write(s, layer, kv, rows[kv][at[s]:at[s + 1]])

    def look():
        lens = cache.seq_len.tolist()
        assert lens == [held.held[s][0][0][0].shape[0] for s in range(n_slots)]
        cu = offsets(lens)
        q = torch.randn(n_slots, H, d, generator=gen, device="cuda").to(dtype)
        for layer in range(n_layers):
            back = S.cache_read(cache, ints(cu), cu[-1], layer=layer)
            for s in range(n_slots):
                for kv in range(2):
                    assert torch.equal(back[kv][cu[s]:cu[s + 1]].double(), held.held[s][layer][kv][0].to(dtype).double())
            out, lse = decode_checked(S, q, cache, held, 20 * layer, 3 * layer, layer=layer)
            # the same by way of a prompt's attention to what was read back
            rows = [s for s in range(n_slots) if lens[s]]
            kw = dict(window=20, sinks=3) if layer else {}
            again = S.prompt_attention(q[rows], *back, ints(offsets([1] * len(rows))), ints(offsets([lens[s] for s in rows])), **kw)
            for i, s in enumerate(rows):
                k, v = (b[cu[s]:cu[s + 1]] for b in back)
                check(again[i:i + 1], None, masked64(q[s:s + 1], k, v, seen_by(1, lens[s], 20 * layer, 3 * layer)), lens[s], d, dtype)

    def fork(parent):
        S.cache_copy_pages(cache, S.cache_fork(cache, ints(parent)))
        for s, p in enumerate(parent):
            if p >= 0:
                held.held[s] = [[[x[0].clone(), x[1].clone()] for x in layer] for layer in held.held[p]]

    step([45, 0, 17, 0, 0, 3])
    look()
    fork([-1, 0, -1, 2, 0, -1])
    look()
    for _ in range(10):
        step([1] * n_slots)
    look()
    S.cache_free(cache, ints([1, 0, 0, 0, 0, 1]))
    held.held[0], held.held[5] = Slots8(1, n_layers, block, G, d).held[0], Slots8(1, n_layers, block, G, d).held[0]
    look()
    S.cache_copy_pages(cache, S.cache_compact(cache))
    look()
    fork([3, -1, -1, -1, -1, 1])
    step([1, 0, 30, 1, 1, 1])
    look()


def test_a_generation_step_in_a_graph(S):
    """reserve, write and attention of a step captured once and replayed, against plain Python."""
    n, G, H, d, page, block = 3, 2, 8, 64, 16, 16
    cache = S.new_cache8(n, 20, page, 6, G, d, block=block)
    held = Slots8(n, 1, block, G, d)
    k, v = (torch.zeros(n, G, d, device="cuda", dtype=BF16) for _ in range(2))
    q, new, cu = torch.zeros(n, H, d, device="cuda", dtype=BF16), ints([1, 1, 0]), ints([0, 1, 2, 2])
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        info = S.cache_reserve(cache, new)
        S.cache_write(cache, k, v, cu, info=info)
        out, lse = S.decode_attention(q, cache, window=30, sinks=2, want_lse=True)
    for i in range(40):
        if i == 25:
            new.copy_(ints([1, 0, 1])), cu.copy_(ints([0, 1, 1, 2]))
        k.copy_(torch.randn_like(k) * (1 + i % 7)), v.copy_(torch.randn_like(v)), q.copy_(torch.randn_like(q))
        graph.replay()
        torch.cuda.synchronize()
        at = cu.tolist()
        for s in range(n):
            for kv, x in enumerate((k, v)):
                held.write(s, 0, kv, x[at[s]:at[s + 1]])
            kk, vv = (held.held[s][0][kv][0] for kv in range(2))
            seen = seen_by(1, kk.shape[0], 30, 2)[0] if kk.shape[0] else slice(0)
            check8(out[s], lse[s], q[s], kk[seen], vv[seen], held.scales_by_token(s, 0, 1)[seen], None, BF16, (i, s))


def test_the_helpers_round_as_the_format_does():
    x = torch.cat([torch.randn(2000, dtype=torch.float64) * 2.0 ** torch.randint(-12, 7, (2000,)), torch.arange(-448, 449).double() / 16]).clamp(-448, 448)
    assert torch.equal(rounded8(x), x.float().to(E4M3).double())
    assert torch.equal(scale_of(torch.tensor([0.0, 448.0, 449.0, 2.0 ** 128])), torch.tensor([2.0 ** -90, 1.0, 2.0, 2.0 ** 120], dtype=torch.float64))
