"""Decode attention over a cache in 8 bits whose scales are 0, NaN or as large as the library writes them, against 64 bits."""
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
                    cache.v_scale[0, p, r // block, g] = (0.0, float("nan"), float("inf"), 1.0)[b % 4]
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
