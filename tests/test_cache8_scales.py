"""Decode attention over a cache in 8 bits whose scales are 0, NaN or far from one, against 64 bits."""
import pytest
import torch

from serve8_helpers import check8, filled_cache8, seen_by
from test_gpu_parity import S  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
NAN = 127  # in e4m3


@pytest.mark.parametrize("H,G,d,dtype", [(8, 2, 128, BF16), (32, 2, 128, BF16), (4, 2, 64, BF16), (12, 1, 256, BF16), (6, 2, 16, BF16), (8, 2, 64, F32),
                                         (2, 2, 128, F32), (12, 1, 256, F32), (24, 2, 32, F32)])
@pytest.mark.parametrize("page,block", [(16, 16), (64, 8), (5, 1)])
def test_tokens_whose_key_scale_is_zero_are_not_there(S, H, G, d, dtype, page, block):
    """Whatever their bytes and their values' scales are, in one kv head alone, and where no other token is."""
    lens = [300, 1, 40, 7, 2000]
    cache, held, led = filled_cache8(S, lens, page, block, G, d, dtype, seed=page)
    q = torch.randn(len(lens), H, d, device="cuda").to(dtype)
    gen = torch.Generator().manual_seed(d)
    left = [[torch.ones(n, dtype=torch.bool) for _ in range(G)] for n in lens]
    for s, n in enumerate(lens):
        for b in range(-(-n // block)):
            for g in range(G):
                if s in (1, 3) or torch.rand(1, generator=gen) < 0.3:  # (two slots lose all of them)
                    p, r = led.table[s][b * block // page], b * block % page
                    cache.k_scale[0, p, r // block, g] = 0.0
                    cache.v_scale[0, p, r // block, g] = (0.0, float("nan"), float("inf"), 1.0, -1.0)[b % 5]
                    for x in (cache.k, cache.v):
                        x.view(torch.uint8)[0, p, r:r + block, g] = (NAN, 255, 126)[b % 3]
                    left[s][g][b * block:(b + 1) * block] = False
    for window, sinks in ((0, 0), (100, 5)):
        out, lse = S.decode_attention(q, cache, window=window, sinks=sinks, want_lse=True)
        for s, n in enumerate(lens):
            for g in range(G):
                at = (left[s][g].cuda() & seen_by(1, n, window, sinks)[0]).nonzero()[:, 0]
                k, v = (held.held[s][0][kv][0][at, g:g + 1] for kv in range(2))
                mine = slice(g * H // G, (g + 1) * H // G)
                check8(out[s, mine], lse[s, mine], q[s, mine], k, v, held.scales_by_token(s, 0, 1)[at, g:g + 1], None, dtype, (s, g, window))


@pytest.mark.parametrize("d,dtype", [(128, BF16), (64, F32), (256, BF16)])
def test_value_scales_of_zero_and_nan(S, d, dtype):
    """A value of scale 0 is 0, and its weight counts; one of scale NaN is NaN, in its head alone."""
    lens, G, H = [300, 16, 2000], 2, 8
    cache, held, led = filled_cache8(S, lens, 16, 16, G, d, dtype)
    q = torch.randn(len(lens), H, d, device="cuda").to(dtype)
    for s, n in enumerate(lens):
        for b in range(-(-n // 16)):
            if b % 3 != 1:
                cache.v_scale[0, led.table[s][b], 0, 0] = 0.0
                held.held[s][0][1][0][16 * b:16 * b + 16, 0] = 0.0
                held.held[s][0][1][1][b, 0] = 0.0
    out, lse = S.decode_attention(q, cache, want_lse=True)
    for s in range(len(lens)):
        k, v = (held.held[s][0][kv][0] for kv in range(2))
        check8(out[s], lse[s], q[s], k, v, held.scales_by_token(s, 0, 1), None, dtype, s)
    assert (out[1, :H // G] == 0).all() and (out[1, H // G:] != 0).any()  # (exactly: nothing of them is left)
    cache.v_scale[0, led.table[0][3], 0, 1] = float("nan")
    got, lse2 = S.decode_attention(q, cache, want_lse=True)
    assert torch.isnan(got[0, H // G:]).all() and torch.equal(lse2, lse)
    assert torch.equal(got[0, :H // G], out[0, :H // G]) and torch.equal(got[1:], out[1:])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("top", [108.0, 60.0, -80.0])
def test_many_small_weights_of_values_far_from_one(S, dtype, top):
    """Scales that the library wrote itself: one token with 2^22.5 times the weight of each of the others, whose sum is what the output is. (All
    2^18 values of 2^108 added up are 2^126: nothing passes fp32.)"""
    n, d, page = 2 ** 18, 64, 1024
    cache = S.new_cache8(1, n // page, page, n // page, 1, d, block=page, dtype=dtype)
    k, v = torch.zeros(n, 1, d, device="cuda"), torch.rand(n, 1, d, device="cuda") / 2 + 0.5
    k[0, 0, 0] = 1.0
    v *= 2.0 ** top
    v[0] *= 2.0 ** -7
    info = S.cache_reserve(cache, torch.tensor([n], dtype=torch.int32, device="cuda"))
    S.cache_write(cache, k.to(dtype), v.to(dtype), torch.tensor([0, n], dtype=torch.int32, device="cuda"), info=info)
    k, v = S.cache_read(cache, torch.tensor([0, n], dtype=torch.int32, device="cuda"), n)
    assert torch.isfinite(v).all()
    q = torch.zeros(1, 2, d, device="cuda")
    q[0, :, 0] = torch.tensor([1.0, 1.0625])
    q = q.to(dtype)
    scale = 22.5 * 0.6931471805599453
    out, lse = S.decode_attention(q, cache, scale=scale, want_lse=True)
    z = cache.v_scale[0, cache.page_table[0].long(), 0].repeat_interleave(page, 0)
    check8(out[0], lse[0], q[0], k, v, z, scale, dtype, top)
