"""A key that is NaN, in a cache of any kind: its head is NaN, output and logarithm, and nothing else is."""
import pytest
import torch

from serve8_helpers import filled_cache8
from serve_helpers import filled_cache
from test_gpu_parity import S  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
LENS, AT = [70, 300, 1, 20000], [13, 299, 0, 7777]  # (the last is dealt to many CTAs)


def looked_at(S, cache, led, d, dtype, set_nan, window):
    H, G = 8, 2
    q = torch.randn(len(LENS), H, d, device="cuda").to(dtype)
    want, ls = S.decode_attention(q, cache, window=window, want_lse=True)
    assert torch.isfinite(want).all() and torch.isfinite(ls).all()
    for s, t in enumerate(AT):
        set_nan(led.table[s][t // cache.page_size], t % cache.page_size)
    out, lse = S.decode_attention(q, cache, window=window, want_lse=True)
    seen = [s for s in range(len(LENS)) if not window or AT[s] >= LENS[s] - window]
    rest = [s for s in range(len(LENS)) if s not in seen]
    assert torch.isnan(out[seen, H // G:]).all() and torch.isnan(lse[seen, H // G:]).all()
    assert torch.equal(out[:, :H // G], want[:, :H // G]) and torch.equal(lse[:, :H // G], ls[:, :H // G])
    assert torch.equal(out[rest], want[rest]) and torch.equal(lse[rest], ls[rest])


@pytest.mark.parametrize("window", [0, 60])
@pytest.mark.parametrize("d,dtype,off", [(128, BF16, 0), (64, F32, 0), (16, BF16, 0), (256, F32, 0), (64, BF16, 1)])
def test_a_key_that_is_nan(S, d, dtype, off, window):
    cache, _, led = filled_cache(S, LENS, 16, 2, d, dtype)
    if off:  # rows that are not aligned
        k, v = (torch.zeros(*x.shape[:4], d + 1, dtype=dtype, device="cuda")[..., 1:] for x in (cache.k, cache.v))
        k.copy_(cache.k), v.copy_(cache.v)
        cache = S.PagedCache(k, v, *led.tensors())

    def set_nan(page, row):
        cache.k[0, page, row, 1, d - 1] = float("nan")

    looked_at(S, cache, led, d, dtype, set_nan, window)


@pytest.mark.parametrize("window", [0, 60])
@pytest.mark.parametrize("d,dtype", [(128, BF16), (64, F32), (16, BF16), (256, F32)])
def test_a_key_that_is_nan_in_8_bits(S, d, dtype, window):
    cache, _, led = filled_cache8(S, LENS, 16, 16, 2, d, dtype)

    def set_nan(page, row):
        cache.k.view(torch.uint8)[0, page, row, 1, d - 1] = 127

    looked_at(S, cache, led, d, dtype, set_nan, window)
