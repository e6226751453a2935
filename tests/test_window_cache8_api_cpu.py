"""Windows, and the paged cache in 8 bits: what the library and the binding refuse, without a GPU."""
import pytest
import torch

from test_api_cpu import S  # noqa: F401  (fixture)
from test_serve_api_cpu import BAD_CACHES, LARGE_CACHES, A, cache, prompt, refused

N = 1 << 40


def cache8(S, block=16, reserved=0, scales=(40, 2, 2, 1), **kw):
    return S.StreamCache8(cache(S, **kw), block, reserved, *scales)


def calls8(S, c):
    return [(S.stream_cache8_write, (c, 0, A, A, 5, 128, 64, A, A, A, None, A, A, A, A, 0)),
            (S.stream_cache8_read, (c, 0, A, A, A, A, A, 5, A, A, A, A, 0)),
            (S.stream_cache8_copy_pages, (c, A, A, A, A, A, A, 3, 0)),
            (S.stream_decode_attention8, (c, 0, 4, 0, 0, A, 256, 64, A, A, A, A, A, A, 0.0, A, None, A, N, 0))]


def calls(S, c):
    return [(S.stream_cache_read, (c, 0, A, A, A, 5, A, A, A, A, 0)),
            (S.stream_decode_window_attention, (c, 0, 4, 7, 2, A, 256, 64, A, A, A, A, 0.0, A, None, A, N, 0))]


@pytest.mark.parametrize("kw", BAD_CACHES + LARGE_CACHES)
def test_caches_that_any_call_refuses(S, kw):
    status = S.STREAM_ERR_INVALID_ARG if kw in BAD_CACHES else S.STREAM_ERR_UNSUPPORTED
    for call, args in calls(S, cache(S, **kw)) + calls8(S, cache8(S, block=1, **kw)):
        refused(S, status, call, *args)


@pytest.mark.parametrize("kw", [dict(block=0), dict(block=-16), dict(block=5), dict(block=32), dict(scales=(0, 2, 2, 1)), dict(scales=(40, 0, 2, 1)),
                                dict(block=8, scales=(80, 4, 0, 1)), dict(scales=(40, 2, 2, 0))])
def test_blocks_and_strides_of_scales(S, kw):
    for call, args in calls8(S, cache8(S, **kw)):
        refused(S, S.STREAM_ERR_INVALID_ARG, call, *args)


def test_pointers(S):
    for call, args in calls(S, cache(S)) + calls8(S, cache8(S)):
        last = len(args) - 3 if "decode" in call.__name__ else -1  # the workspace
        for i, x in enumerate(args):
            if x is A:
                for bad in (None, A + 1):
                    if bad and call is not S.stream_cache_read and i in {S.stream_cache8_write: (11, 12), S.stream_cache8_read: (2, 3),
                                                                         S.stream_cache8_copy_pages: (1, 2), S.stream_decode_attention8: (8, 9)}.get(call, ()):
                        continue  # (bytes lie anywhere)
                    refused(S, S.STREAM_ERR_WORKSPACE if i == last else S.STREAM_ERR_INVALID_ARG, call, *(bad if j == i else y for j, y in enumerate(args)))
        if last > 0:
            refused(S, S.STREAM_ERR_WORKSPACE, call, *(64 if j == last + 1 else y for j, y in enumerate(args)))


def test_layers_totals_heads_and_scales(S):
    c, c8 = cache(S), cache8(S)
    for layer in (-1, 3):
        for call, args in calls(S, c) + calls8(S, c8):
            if call is not S.stream_cache8_copy_pages:
                refused(S, S.STREAM_ERR_INVALID_ARG, call, args[0], layer, *args[2:])
    for total in (-1, 2 ** 31):
        refused(S, S.STREAM_ERR_INVALID_ARG, S.stream_cache_read, c, 0, A, A, A, total, A, A, A, A, 0)
        refused(S, S.STREAM_ERR_INVALID_ARG, S.stream_cache8_read, c8, 0, A, A, A, A, A, total, A, A, A, A, 0)
    for total, st, sh in ((-1, 128, 64), (2 ** 31, 128, 64), (5, 63, 64), (5, 128, 0)):
        refused(S, S.STREAM_ERR_INVALID_ARG, S.stream_cache8_write, c8, 0, A, A, total, st, sh, A, A, A, A, A, A, A, A, 0)
    refused(S, S.STREAM_ERR_INVALID_ARG, S.stream_cache8_copy_pages, c8, A, A, A, A, A, A, -1, 0)
    for heads, window, sinks, st, sh, scale in ((3, 1, 0, 256, 64, 0.0), (0, 1, 0, 256, 64, 0.0), (4, -1, 0, 256, 64, 0.0), (4, 5, -1, 256, 64, 0.0), (4, 5, 0, 63, 64, 0.0),
                                                (4, 5, 0, 256, 63, 0.0), (4, 5, 0, 256, 64, float("inf")), (4, 5, 0, 256, 64, float("nan"))):
        refused(S, S.STREAM_ERR_INVALID_ARG, S.stream_decode_attention8, c8, 0, heads, window, sinks, A, st, sh, A, A, A, A, A, A, scale, A, None, A, N, 0)
        refused(S, S.STREAM_ERR_INVALID_ARG, S.stream_decode_window_attention, c, 0, heads, window, sinks, A, st, sh, A, A, A, A, scale, A, None, A, N, 0)
    refused(S, S.STREAM_ERR_INVALID_ARG, S.stream_decode_window_attention, c, 0, 4, 0, 3, A, 256, 64, A, A, A, A, 0.0, A, None, A, N, 0)
    # nothing to do
    S.stream_cache_read(c, 0, None, None, A, 0, A, A, None, None, 0)
    S.stream_cache8_read(c8, 0, None, None, A, A, A, 0, A, A, None, None, 0)
    S.stream_cache8_write(c8, 0, None, None, 0, 128, 64, A, A, A, None, None, None, A, A, 0)
    S.stream_cache8_copy_pages(c8, None, None, A, A, None, None, 0, 0)


def test_windows_of_prompts(S):
    good = [A, A, A, A, A, 0.0, A, None, 0]
    for window, sinks, kw in ((0, 0, {}), (-1, 0, {}), (5, -1, {}), (5, 0, dict(causal=0)), (5, 0, dict(n_q_heads=3)), (5, 0, dict(dtype=7))):
        refused(S, S.STREAM_ERR_INVALID_ARG, S.stream_prompt_window_attention, prompt(S, **kw), window, sinks, *good)
    refused(S, S.STREAM_ERR_UNSUPPORTED, S.stream_prompt_window_attention, prompt(S, d=96, q_stride_h=96, kv_stride_h=96), 5, 0, *good)
    for i in (0, 1, 2, 3, 4, 6):
        for bad in (None, A + 1):
            refused(S, S.STREAM_ERR_INVALID_ARG, S.stream_prompt_window_attention, prompt(S), 5, 0, *(bad if j == i else x for j, x in enumerate(good)))
    S.stream_prompt_window_attention(prompt(S, total_q=0), 5, 2, None, None, None, A, A, 0.0, None, None, 0)


class OnGpu(torch.Tensor):
    is_cuda = True


def tensors(block=16, dtype=torch.float8_e4m3fn):
    k, z = torch.zeros(1, 4, 16, 2, 64).to(dtype).as_subclass(OnGpu), torch.zeros(1, 4, 16 // block, 2)
    ledger = torch.full((2, 3), -1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    return k, z, ledger


def test_the_binding_refuses(S):
    k, z, ledger = tensors()
    with pytest.raises(ValueError):
        S.PagedCache8(k.as_subclass(torch.Tensor), k.as_subclass(torch.Tensor), z, z, *ledger)  # no CUDA tensors
    for args, kw in (((k.view(torch.uint8), k, z, z), {}), ((k, k, z[:, :, :, :1], z), {}), ((k, k, z, z.double()), {}), ((k, k, z, z.transpose(0, 1)), {}),
                     ((k, k, torch.zeros(1, 4, 3, 2), torch.zeros(1, 4, 3, 2)), {}), ((k, k, z[0], z[0]), {}), ((k, k, z, z), dict(dtype=torch.float16)),
                     ((k, k, torch.zeros(1, 4, 0, 2), torch.zeros(1, 4, 0, 2)), {}), ((k, k[:, :3], z, z), {})):
        with pytest.raises(ValueError):
            S.PagedCache8(*args, *ledger, **kw)
    with pytest.raises(ValueError):
        S.new_cache8(2, 4, 16, 2, 2, 64, block=5, device="cpu")
    c = S.PagedCache8(k, k, z, z, *ledger)
    assert c.block == 16 and c.dtype is torch.bfloat16
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    for kw in (dict(window=-1), dict(sinks=2), dict(window=3, sinks=-1)):
        with pytest.raises(ValueError):
            S.decode_attention(q, c, **kw)
        with pytest.raises(ValueError):
            S.prompt_attention(*(x.as_subclass(OnGpu) for x in (q, q, q)), torch.zeros(2, dtype=torch.int32).as_subclass(OnGpu), **kw)
    with pytest.raises(ValueError):
        S.prompt_attention(*(x.as_subclass(OnGpu) for x in (q, q, q)), torch.zeros(2, dtype=torch.int32).as_subclass(OnGpu), window=3, causal=False)
    with pytest.raises(ValueError):
        S.decode_attention(q.float(), c)
    cu = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        S.cache_write(c, q[:, :2].float(), q[:, :2].float(), cu)
    for kw in (dict(layer=1), dict(out=(q, q)), dict(cu=cu[:2]), dict(total=-1), dict(total=2 ** 31)):
        with pytest.raises(ValueError):
            S.cache_read(**dict(dict(cache=c, cu=cu, total=2), **kw))


@pytest.mark.parametrize("what", ["decode", "write", "copy", "read"])
def test_a_stream_of_another_device_is_refused(S, monkeypatch, what):
    class Stream:
        device, cuda_stream = torch.device("cuda", 1), 12345

    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    k, z, ledger = tensors()
    c = S.PagedCache8(k, k, z, z, *ledger)
    q, cu = torch.zeros(2, 4, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    moves = S.CacheMoves(torch.zeros(1, 2, dtype=torch.int32), torch.zeros(4, dtype=torch.int32))
    calls = dict(decode=lambda st: S.decode_attention(q, c, window=3, stream=st), write=lambda st: S.cache_write(c, q[:, :2], q[:, 2:], cu, stream=st),
                 copy=lambda st: S.cache_copy_pages(c, moves, stream=st), read=lambda st: S.cache_read(c, cu, 2, stream=st))
    with pytest.raises(ValueError, match="stream"):
        calls[what](Stream())
