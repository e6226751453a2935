"""The workspace of decode attention: as large as two pieces of an owner for each CTA, for caches of every kind, and nothing behind it is touched."""
import random

import pytest
import torch

from serve8_helpers import check8, filled_cache8, masked64, seen_by
from serve_helpers import check, filled_cache
from test_api_cpu import S  # noqa: F401  (fixture)
from test_serve_api_cpu import cache as cache_struct

BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("d", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("dtype", [0, 1])
def test_its_size(S, d, dtype):
    c = cache_struct(S, d=d, dtype=dtype, stride_h=d, stride_t=2 * d, stride_p=32 * d, stride_l=32 * d * 20)
    for heads in (2, 8, 16, 64):
        n = S.stream_decode_workspace_bytes(c, heads)
        assert 0 < n <= 320 * 2 * 16 * (d + 2) * 4 + 32768, n


@pytest.mark.gpu
@pytest.mark.parametrize("H,G", [(32, 2), (17, 1), (8, 2), (40, 2)])
@pytest.mark.parametrize("d,dtype", [(128, BF16), (256, F32), (256, BF16), (64, F32)])
@pytest.mark.parametrize("eight", [True, False])
def test_what_lies_behind_it_stays(S, H, G, d, dtype, eight):
    """Many short slots beside long ones: most warps meet an owner's end, some of them several."""
    rng = random.Random(d + H)
    for lens in ([rng.randint(0, 200) for _ in range(150)], [5000, 33, 0, 31, 64, 2000], [rng.choice([1, 32, 33, 700]) for _ in range(60)]):
        make = (lambda: filled_cache8(S, lens, 32, 16, G, d, dtype)) if eight else (lambda: filled_cache(S, lens, 32, G, d, dtype))
        cache, held, _ = make()
        q = torch.randn(len(lens), H, d, device="cuda").to(dtype)
        need = S.stream_decode_workspace_bytes(cache.struct, H)
        room = torch.full((256 + need + 4096,), 77, dtype=torch.uint8, device="cuda")
        for window in (0, 90):
            out, lse = S.decode_attention(q, cache, window=window, want_lse=True, workspace=room[256:256 + need])
            torch.cuda.synchronize()
            assert (room[:256] == 77).all() and (room[256 + need:] == 77).all()
            for s in range(0, len(lens), 1 if len(lens) < 10 else 7):
                seen = seen_by(1, lens[s], window, 0)
                if eight:
                    at = seen[0]
                    k, v = (held.held[s][0][kv][0][at] for kv in range(2))
                    check8(out[s], lse[s], q[s], k, v, held.scales_by_token(s, 0, 1)[at], None, dtype, (s, window))
                else:
                    k, v = (x[0] for x in held[s])
                    check(out[s:s + 1], lse[s:s + 1].T, masked64(q[s:s + 1], k, v, seen), lens[s], d, dtype, (s, window))
