"""Dense attention and the paged cache: what the library and the binding refuse, without a GPU."""
import os
import re

import pytest
import torch

import paper_2510_19875_b200
from test_api_cpu import S  # noqa: F401  (fixture)

CSRC = os.path.join(os.path.dirname(paper_2510_19875_b200.__file__), "csrc")
A = 4096  # an address that nothing is read from: the calls below are refused before anything is launched


def prompt(S, **kw):
    base = dict(n_seqs=2, n_q_heads=4, n_kv_heads=2, d=64, total_q=100, total_k=100, causal=1, dtype=S.STREAM_BF16, q_stride_t=256,
                q_stride_h=64, kv_stride_t=128, kv_stride_h=64)
    base.update(kw)
    return S.StreamPrompt(**base)


def cache(S, **kw):
    base = dict(n_slots=4, n_pages=20, page_size=16, max_pages=8, n_kv_heads=2, d=64, n_layers=3, dtype=S.STREAM_BF16,
                stride_l=20 * 16 * 128, stride_p=16 * 128, stride_t=128, stride_h=64)
    base.update(kw)
    return S.StreamCache(**base)


def refused(S, status, call, *args):
    with pytest.raises(S.StreamError) as e:
        call(*args)
    assert e.value.status == status
    assert S.stream_last_error() != ""


@pytest.mark.parametrize("kw", [dict(n_seqs=0), dict(n_q_heads=3), dict(n_kv_heads=0), dict(dtype=5), dict(causal=2), dict(total_q=-1), dict(total_k=-1),
                                dict(q_stride_t=63), dict(q_stride_h=1), dict(kv_stride_t=0), dict(kv_stride_h=-64), dict(d=0), dict(d=-64)])
def test_invalid_prompts(S, kw):
    refused(S, S.STREAM_ERR_INVALID_ARG, S.stream_prompt_attention, prompt(S, **kw), A, A, A, A, A, 0.0, A, None, 0)


@pytest.mark.parametrize("kw", [dict(d=96, q_stride_h=96, kv_stride_h=96), dict(total_q=2 ** 31), dict(total_k=2 ** 31), dict(n_seqs=2 ** 25), dict(n_q_heads=2 ** 18)])
def test_unsupported_prompts(S, kw):
    refused(S, S.STREAM_ERR_UNSUPPORTED, S.stream_prompt_attention, prompt(S, **kw), A, A, A, A, A, 0.0, A, None, 0)


def test_prompt_pointers(S):
    good = [A, A, A, A, A, 0.0, A, None]
    for i in (0, 1, 2, 3, 4, 6):
        refused(S, S.STREAM_ERR_INVALID_ARG, S.stream_prompt_attention, prompt(S), *(None if j == i else x for j, x in enumerate(good)), 0)
        refused(S, S.STREAM_ERR_INVALID_ARG, S.stream_prompt_attention, prompt(S), *(A + 1 if j == i else x for j, x in enumerate(good)), 0)
    for scale in (float("inf"),):
        refused(S, S.STREAM_ERR_INVALID_ARG, S.stream_prompt_attention, prompt(S), A, A, A, A, A, scale, A, None, 0)
    S.stream_prompt_attention(prompt(S, total_q=0), None, None, None, A, A, 0.0, None, None, 0)  # nothing to do
    # a stride that separates nothing does not matter
    S.stream_prompt_attention(prompt(S, total_q=0, q_stride_t=0, n_kv_heads=1, kv_stride_h=0, total_k=1, kv_stride_t=0), None, None, None, A, A, 0.0, None, None, 0)


BAD_CACHES = [dict(n_slots=0), dict(n_pages=0), dict(page_size=0), dict(max_pages=-1), dict(n_kv_heads=0), dict(n_layers=0), dict(d=0), dict(dtype=2),
              dict(stride_l=0), dict(stride_p=-1), dict(stride_t=63), dict(stride_h=0)]
LARGE_CACHES = [dict(d=48), dict(n_slots=2 ** 20, max_pages=2 ** 12), dict(page_size=2 ** 20, max_pages=2 ** 12), dict(n_pages=2 ** 30 + 1), dict(page_size=2 ** 24, max_pages=1)]


def every_call(S, c):
    n = 1 << 40
    return [(S.stream_cache_reserve, (c, A, A, A, A, A, A, n, 0)), (S.stream_cache_fork, (c, A, A, A, A, A, A, A, n, 0)),
            (S.stream_cache_free, (c, A, A, A, A, A, A, n, 0)), (S.stream_cache_compact, (c, A, A, A, A, A, A, n, 0)),
            (S.stream_cache_copy_pages, (c, A, A, A, A, 3, 0)), (S.stream_cache_write, (c, 0, A, A, 5, 128, 64, A, A, A, None, A, A, 0)),
            (S.stream_decode_attention, (c, 0, 4, A, 256, 64, A, A, A, A, 0.0, A, None, A, n, 0))]


@pytest.mark.parametrize("kw", BAD_CACHES)
def test_invalid_caches(S, kw):
    c = cache(S, **kw)
    assert S.stream_cache_workspace_bytes(c) == 0 and S.stream_decode_workspace_bytes(c, 4) == 0
    for call, args in every_call(S, c):
        refused(S, S.STREAM_ERR_INVALID_ARG, call, *args)


@pytest.mark.parametrize("kw", LARGE_CACHES)
def test_unsupported_caches(S, kw):
    c = cache(S, **kw)
    assert S.stream_cache_workspace_bytes(c) == 0 and S.stream_decode_workspace_bytes(c, 4) == 0
    for call, args in every_call(S, c):
        refused(S, S.STREAM_ERR_UNSUPPORTED, call, *args)


def test_pointers_and_workspaces(S):
    c = cache(S)
    assert S.stream_cache_workspace_bytes(c) >= 4 * (4 + 20) and S.stream_decode_workspace_bytes(c, 4) > 256
    for call, args in every_call(S, c):
        name = call.__name__
        for i, x in enumerate(args):
            if x == A and not isinstance(x, bool):
                last = call in (S.stream_cache_reserve, S.stream_cache_fork, S.stream_cache_free, S.stream_cache_compact, S.stream_decode_attention) and i == len(args) - 3
                for bad in (None, A + 1):  # missing; aligned to nothing
                    refused(S, S.STREAM_ERR_WORKSPACE if last else S.STREAM_ERR_INVALID_ARG, call, *(bad if j == i else y for j, y in enumerate(args)))
                if last:
                    for n in (0, 64):
                        refused(S, S.STREAM_ERR_WORKSPACE, call, *(n if j == i + 1 else y for j, y in enumerate(args)))
        assert name.startswith("stream_")
    refused(S, S.STREAM_ERR_INVALID_ARG, S.stream_cache_copy_pages, c, A, A, A, A, -1, 0)
    S.stream_cache_copy_pages(c, None, None, None, None, 0, 0)
    for layer in (-1, 3):
        refused(S, S.STREAM_ERR_INVALID_ARG, S.stream_cache_write, c, layer, A, A, 5, 128, 64, A, A, A, A, A, A, 0)
        refused(S, S.STREAM_ERR_INVALID_ARG, S.stream_decode_attention, c, layer, 4, A, 256, 64, A, A, A, A, 0.0, A, None, A, 1 << 40, 0)
    for total, st, sh in ((-1, 128, 64), (2 ** 31, 128, 64), (5, 63, 64), (5, 128, 0)):
        refused(S, S.STREAM_ERR_INVALID_ARG, S.stream_cache_write, c, 0, A, A, total, st, sh, A, A, A, A, A, A, 0)
    S.stream_cache_write(c, 0, None, None, 0, 128, 64, A, A, A, None, None, None, 0)
    refused(S, S.STREAM_ERR_INVALID_ARG, S.stream_cache_write, c, 0, A, A, 5, 128, 64, A, A, A, A + 2, A, A, 0)
    for heads, st, sh, scale in ((3, 256, 64, 0.0), (0, 256, 64, 0.0), (4, 63, 64, 0.0), (4, 256, 63, 0.0), (4, 256, 64, float("inf"))):
        refused(S, S.STREAM_ERR_INVALID_ARG, S.stream_decode_attention, c, 0, heads, A, st, sh, A, A, A, A, scale, A, None, A, 1 << 40, 0)
    assert S.stream_decode_workspace_bytes(c, 3) == 0 and S.stream_decode_workspace_bytes(c, 0) == 0


def test_cpu_tensors_are_refused(S):
    q, cu = torch.zeros(4, 2, 64), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        S.prompt_attention(q, q, q, cu)
    k = torch.zeros(1, 2, 4, 2, 64)
    with pytest.raises(ValueError):
        S.PagedCache(k, k, torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32))


EARLY = sorted(f for f in os.listdir(CSRC) if f.endswith(".cu") and "launch_early(" in open(os.path.join(CSRC, f)).read())


@pytest.mark.parametrize("name", EARLY + ["serve_common.cuh", "decode.cuh"])
def test_kernels_that_begin_early_read_no_memory_as_constant(name):
    """As the other programmatic dependents: they live while the kernel before them still writes."""
    assert {"prompt_tc.cu", "prompt_generic.cu", "decode.cu", "decode_warp.cu", "prompt_mma.cu", "cache_ledger.cu", "cache_copy.cu"} <= set(EARLY)
    text = re.sub(r"//.*", "", open(os.path.join(CSRC, name)).read())
    assert not re.findall(r"__ldg\s*\(|ld\.global\.nc", text)
    assert not re.findall(r"const [\w: ]+\*\s*__restrict__", text)


def test_largest_sizes(S):
    """As many tokens and slots as 32 bits count with a tile's rows added, and one more."""
    most = 2 ** 31 - 4096
    for kw in (dict(total_q=most + 1), dict(total_k=most + 1)):
        refused(S, S.STREAM_ERR_UNSUPPORTED, S.stream_prompt_attention, prompt(S, **kw), A, A, A, A, A, 0.0, A, None, 0)
    S.stream_prompt_attention(prompt(S, total_q=0, total_k=most), None, None, None, A, A, 0.0, None, None, 0)  # nothing to do
    for good, bad in ((dict(max_pages=most, page_size=1, n_slots=1), dict(max_pages=most + 1, page_size=1, n_slots=1)),
                      (dict(n_slots=2 ** 30, max_pages=1), dict(n_slots=2 ** 30 + 1, max_pages=1))):
        assert S.stream_cache_workspace_bytes(cache(S, **good)) > 0
        c = cache(S, **bad)
        assert S.stream_cache_workspace_bytes(c) == 0 and S.stream_decode_workspace_bytes(c, 4) == 0
        for call, args in every_call(S, c):
            refused(S, S.STREAM_ERR_UNSUPPORTED, call, *args)


@pytest.mark.parametrize("name,threads,rows,per_piece,dims", [("prompt_mma.cu", 256, 128, 8, (16, 32, 64, 128, 256)), ("prompt_f32.cu", 128, 64, 4, (16, 32, 64, 128))])
def test_output_in_the_place_of_q_waits_for_every_warps_copies(name, threads, rows, per_piece, dims):
    """A tile without keys runs no barrier in its key loop: one has to stand between the copies of Q, most of which threads of
    other warps make, and the output that takes Q's place."""
    others = {}
    for d in dims:
        pieces = d // per_piece  # piece i, of row i / pieces, is thread i % threads' to copy; 16 rows are a warp's
        others[d] = sum(i % threads // 32 != i // pieces // 16 for i in range(rows * pieces))
    assert max(others.values()) > 0
    text = re.sub(r"//.*", "", open(os.path.join(CSRC, name)).read())
    assert re.search(r"i % kPieces.*\n(?:.*\n){1,3}.*cp_async16\(q_s", text)  # (as modelled here)
    behind = text[text.index("cp_async_wait<0>()"):]  # the first is behind the loop
    output = re.search(r"sm\.q \+", behind)
    assert "__syncthreads()" in behind[:output.start()]


@pytest.mark.parametrize("what", ["prompt", "decode", "reserve", "fork", "free", "compact", "write", "copy"])
def test_a_stream_of_another_device_is_refused(S, monkeypatch, what):
    """By every call, before anything is launched or allocated. (Device cpu stands for the tensors' own.)"""
    class Stream:
        device, cuda_stream = torch.device("cuda", 1), 12345

    class OnGpu(torch.Tensor):
        is_cuda = True

    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    ints = lambda *x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    k = torch.zeros(1, 4, 4, 2, 64)
    q, one, cu = torch.zeros(2, 4, 64), ints(1, 0), ints(0, 1, 1)
    c = object.__new__(S.PagedCache)
    c.device, c.k, c.v, c.page_table, c.seq_len, c.ref_count = k.device, k, k, ints(-1, -1).view(2, 1), ints(0, 0), ints(0, 0, 0, 0)
    c.n_layers, c.n_pages, c.page_size, c.n_kv_heads, c.d, c.n_slots, c.max_pages, c._p = 1, 4, 4, 2, 64, 2, 1, None
    t = lambda x: x.as_subclass(OnGpu)  # noqa: E731
    calls = dict(prompt=lambda st: S.prompt_attention(t(q), t(q), t(q), t(cu), stream=st), decode=lambda st: S.decode_attention(q, c, stream=st),
                 reserve=lambda st: S.cache_reserve(c, one, stream=st), fork=lambda st: S.cache_fork(c, one, stream=st),
                 free=lambda st: S.cache_free(c, one, stream=st), compact=lambda st: S.cache_compact(c, stream=st),
                 write=lambda st: S.cache_write(c, q[:, :2], q[:, 2:], cu, stream=st),
                 copy=lambda st: S.cache_copy_pages(c, S.CacheMoves(ints(-1, -1).view(1, 2), ints(1, 0, 0, 0)), stream=st))
    with pytest.raises(ValueError, match="stream"):
        calls[what](Stream())


@pytest.mark.parametrize("scale", [float("nan"), float("inf"), 3.4e38, 2.36e38])  # (the last, times log2(e), is 2^128 and a little)
def test_scales_whose_logits_fp32_does_not_hold(S, scale):
    refused(S, S.STREAM_ERR_INVALID_ARG, S.stream_prompt_attention, prompt(S), A, A, A, A, A, scale, A, None, 0)
    refused(S, S.STREAM_ERR_INVALID_ARG, S.stream_decode_attention, cache(S), 0, 4, A, 256, 64, A, A, A, A, scale, A, None, A, 1 << 40, 0)
