"""Windows of prompts at the kernels' borders: sinks that just fill a shared tile or one of their own, and more items than a CTA has room to list."""
import pytest
import torch

from serve8_helpers import masked64
from serve_helpers import check, ints
from test_dense_attention import inputs
from test_gpu_parity import S  # noqa: F401  (fixture)
from test_window_attention import run

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("H,G,d,dtype", [(8, 2, 128, BF16), (7, 1, 64, BF16), (4, 2, 256, BF16), (2, 1, 64, F32), (2, 1, 256, F32)])
@pytest.mark.parametrize("sinks", [15, 16, 17, 31, 32, 33, 64, 127, 128, 129, 256])
def test_sinks(S, H, G, d, dtype, sinks):
    q, k, v, cu_q, cu_k = inputs(H, G, d, [900, 40, 333], [900, 800, 333], dtype, seed=sinks)
    for window in (1, 100, 128, 257, 500):
        run(S, q, k, v, cu_q, cu_k, window, sinks)


@pytest.mark.parametrize("window,sinks", [(200, 16), (130, 40), (0, 0)])
def test_more_items_than_a_cta_lists(S, window, sinks):
    """A kv head of 128 query heads has a token a tile, so that the items of a CTA are many, of one sequence and of several."""
    H, d = 128, 64
    for lens in ([21000], [9000, 3, 0, 11000, 1000]):
        cu = [0]
        for n in lens:
            cu.append(cu[-1] + n)
        total = cu[-1]
        q, k, v = (torch.randn(total, h, d, device="cuda", dtype=BF16) for h in (H, 1, 1))
        out, lse = S.prompt_attention(q, k, v, ints(cu), window=window, sinks=sinks, want_lse=True)
        torch.cuda.synchronize()
        S.stream_check_device_status()
        for a, b in zip(cu, cu[1:]):
            for at in {a, a + 17, a + 150, (a + b) // 2, b - 2, b - 1}:
                if not a <= at < b:
                    continue
                j = torch.arange(a, at + 1, device="cuda")
                keys = j[(j > at - window) | (j < a + sinks)] if window else j
                want = masked64(q[at:at + 1], k[keys], v[keys], torch.ones(1, len(keys), dtype=torch.bool, device="cuda"))
                check(out[at:at + 1], lse[:, at:at + 1], want, len(keys), d, BF16, at)
