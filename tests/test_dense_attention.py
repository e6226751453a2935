"""Dense attention of packed prompts against 64 bits: every kernel, its ragged ends, masks that leave rows empty, strides."""
import pytest
import torch

from serve_helpers import attention64, check, ints, offsets
from test_gpu_parity import S  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def inputs(H, G, d, lens_q, lens_k, dtype, *, behind=0, seed=0, sink=True):
    gen = torch.Generator("cuda").manual_seed(seed)
    cu_q, cu_k = offsets(lens_q), offsets(lens_k)
    q = torch.randn(cu_q[-1] + behind, H, d, generator=gen, device="cuda")
    k, v = (torch.randn(cu_k[-1] + behind, G, d, generator=gen, device="cuda") for _ in range(2))
    if sink:  # a first key that stands out, and later ones that outgrow it
        for a, b in zip(cu_k, cu_k[1:]):
            if b > a:
                k[a] *= 3
                k[(a + b) // 2] *= 5
    q, k, v = q.to(dtype), k.to(dtype), v.to(dtype)
    k[cu_k[-1]:] = float("nan")
    v[cu_k[-1]:] = float("nan")
    return q, k, v, cu_q, cu_k


def want(q, k, v, cu_q, cu_k, causal, scale=None):
    parts = []
    for s in range(len(cu_q) - 1):
        a, b, x, y = cu_q[s], cu_q[s + 1], cu_k[s], cu_k[s + 1]
        parts.append(attention64(q[a:b], k[x:y], v[x:y], (y - x) - (b - a) if causal else None, scale))
    return tuple(torch.cat([p[i] for p in parts], 1 if i == 1 else 0) for i in range(4))


def run(S, q, k, v, cu_q, cu_k, causal, **kw):
    n, H, d = cu_q[-1], q.shape[1], q.shape[2]
    out = torch.full((q.shape[0], H, d), 7.0, dtype=q.dtype, device="cuda")
    lse = torch.full((H, q.shape[0]), 7.0, device="cuda")
    S.prompt_attention(q, k, v, ints(cu_q), ints(cu_k), causal=causal, out=out, lse_out=lse, **kw)
    torch.cuda.synchronize()
    S.stream_check_device_status()
    assert (out[n:] == 7).all() and (lse[:, n:] == 7).all()  # rows of no sequence
    check(out[:n], lse[:, :n], want(q, k, v, cu_q, cu_k, causal, kw.get("scale")), max([b - a for a, b in zip(cu_k, cu_k[1:])]), d, q.dtype)
    return out, lse


SHAPES = [(1, 1, 128), (8, 2, 128), (7, 1, 64), (28, 4, 128), (6, 2, 64), (16, 16, 128), (33, 1, 64)]
LENS = [
    ([1], [1]), ([128], [128]), ([129], [129]), ([5, 0, 300, 1], [5, 0, 300, 1]),   # one token, whole tiles, one beyond, an empty one
    ([3, 40], [300, 41]),                                                            # keys before the first query
    ([200, 7, 150], [60, 0, 149]),                                                   # queries that see nothing, no keys at all
]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("H,G,d", SHAPES)
def test_tensor_core_kernel(S, H, G, d, lens, causal):
    q, k, v, cu_q, cu_k = inputs(H, G, d, *lens, BF16, behind=5, seed=H + d)
    run(S, q, k, v, cu_q, cu_k, causal)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("H,G,d,dtype", [(1, 1, 64, F32), (8, 2, 128, F32), (6, 2, 32, F32), (3, 1, 16, F32), (2, 1, 256, F32),
                                         (8, 2, 256, BF16), (6, 2, 32, BF16), (7, 1, 16, BF16), (300, 2, 64, BF16)])
def test_other_kernels(S, H, G, d, dtype, lens, causal):
    q, k, v, cu_q, cu_k = inputs(H, G, d, *lens, dtype, behind=5, seed=H + d)
    run(S, q, k, v, cu_q, cu_k, causal)


@pytest.mark.parametrize("H,G,d,n,dtype", [(8, 2, 128, 3001, BF16), (4, 4, 64, 2500, BF16), (2, 1, 64, 2500, F32), (2, 2, 128, 1999, F32), (4, 1, 256, 1500, BF16)])
def test_long_sequences(S, H, G, d, n, dtype):
    q, k, v, cu_q, cu_k = inputs(H, G, d, [n, 77], [n, 500], dtype, seed=n)
    run(S, q, k, v, cu_q, cu_k, True)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("H,G,d,lens_q,lens_k", [
    (28, 4, 128, [700, 1500, 0, 333, 64, 2000, 1, 129], [700, 1600, 5, 333, 2000, 2000, 1300, 0]),  # put in the order of their keys
    (8, 8, 64, [600, 600, 600, 1], [600, 599, 40, 900]),
    (128, 1, 64, [5000, 300], [5000, 300]),                                                          # too many to be put in order
])
def test_more_items_than_ctas(S, H, G, d, lens_q, lens_k, causal):
    q, k, v, cu_q, cu_k = inputs(H, G, d, lens_q, lens_k, BF16, behind=7, seed=H)
    run(S, q, k, v, cu_q, cu_k, causal)


@pytest.mark.parametrize("n", [70_000, 1_200_000])
def test_keys_of_more_than_the_cache_holds_and_a_kernel_of_seconds(S, n):
    """Three kv heads of eight, then one, are walked at a time. Waits have a limit of about a second, but some roles of the tensor-core
    kernel wait for items far ahead: a short prompt behind one of a million tokens and more."""
    m, d = 77, 128
    q, k, v = (torch.randn(n + m, h, d, device="cuda", dtype=BF16) for h in (8, 8, 8))
    out, lse = S.prompt_attention(q, k, v, ints([0, n, n + m]), want_lse=True)
    torch.cuda.synchronize()
    S.stream_check_device_status()
    check(out[n:], lse[:, n:], attention64(q[n:], k[n:], v[n:], 0), m, d, BF16)
    for at in (0, 1000, n // 2 + 1, n - 3):
        some = attention64(q[at:at + 3], k[:at + 3], v[:at + 3], at)
        check(out[at:at + 3], lse[:, at:at + 3], some, at + 3, d, BF16)


def test_many_sequences(S):
    """More sequences than the tensor-core kernel takes in one launch, of all lengths from none."""
    lens = [i % 23 for i in range(1300)]
    q, k, v, cu_q, cu_k = inputs(4, 2, 64, lens, lens, BF16, behind=3)
    run(S, q, k, v, cu_q, cu_k, True)
    run(S, q.float(), k.float(), v.float(), cu_q, cu_k, True)


def test_logits_that_outgrow_their_reference(S):
    """Rows whose largest logits come late and are larger by far more than the kernel lets its reference lag behind."""
    q, k, v, cu_q, cu_k = inputs(4, 2, 128, [700], [700], BF16, sink=False)
    k *= (torch.arange(700, device="cuda")[:, None, None] / 60).bfloat16()
    run(S, q, k, v, cu_q, cu_k, True)
    run(S, q, k.flip(0).contiguous(), v, cu_q, cu_k, False)


@pytest.mark.parametrize("scale", [0.01, 0.5])
def test_scale(S, scale):
    for d, dtype in ((128, BF16), (64, F32)):
        q, k, v, cu_q, cu_k = inputs(4, 2, d, [300], [300], dtype)
        run(S, q, k, v, cu_q, cu_k, True, scale=scale)


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 64)])
def test_strides(S, dtype, d):
    """Heads outside tokens, parts of wider rows, and rows that are not aligned to 16 bytes (another kernel)."""
    q, k, v, cu_q, cu_k = inputs(8, 2, d, [150, 90], [150, 90], dtype)
    a = run(S, q, k, v, cu_q, cu_k, True)
    heads_outside = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v)]
    b = run(S, *heads_outside, cu_q, cu_k, True)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    wide = torch.zeros(240, 12, 2 * d, dtype=dtype, device="cuda")
    wide[:, :8, :d], wide[:, 8:10, :d], wide[:, 10:, d:] = q, k, v
    b = run(S, wide[:, :8, :d], wide[:, 8:10, :d], wide[:, 10:, d:], cu_q, cu_k, True)
    assert torch.equal(a[0], b[0])
    odd = torch.zeros(240, 12, d + 1, dtype=dtype, device="cuda")
    odd[:, :8, 1:], odd[:, 8:10, 1:], odd[:, 10:, 1:] = q, k, v
    run(S, odd[:, :8, 1:], odd[:, 8:10, 1:], odd[:, 10:, 1:], cu_q, cu_k, True)


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 256), (F32, 64)])
def test_what_lies_outside_a_sequence_does_not_matter(S, dtype, d):
    q, k, v, cu_q, cu_k = inputs(4, 2, d, [100, 60, 30], [100, 60, 30], dtype, behind=140)
    a = run(S, q, k, v, cu_q, cu_k, True)
    k2, v2, q2 = k.clone(), v.clone(), q.clone()
    for x in (k2, v2, q2):
        x[:100] = float("inf")
        x[160:] = float("nan")
    out, lse = S.prompt_attention(q2, k2, v2, ints(cu_q), ints(cu_k), want_lse=True)
    assert torch.equal(out[100:160], a[0][100:160]) and torch.equal(lse[:, 100:160], a[1][:, 100:160])


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (F32, 32)])
def test_offsets_that_cannot_be_stay_inside(S, dtype, d):
    """Offsets outside the tensors count as the nearest inside, an end before its beginning is an empty sequence."""
    q, k, v, cu_q, cu_k = inputs(4, 2, d, [200], [200], dtype)
    out, lse = S.prompt_attention(q, k, v, ints([-50, 2 ** 31 - 1]), ints([-2 ** 31, 900]), want_lse=True)
    check(out, lse, want(q, k, v, [0, 200], [0, 200], True), 200, d, dtype)
    out = torch.full_like(q, 7.0)
    S.prompt_attention(q, k, v, ints([150, 50, 60]), ints([0, 100, 200]), out=out)
    torch.cuda.synchronize()
    S.stream_check_device_status()
    ref = want(q[50:60], k[100:], v[100:], [0, 10], [0, 100], True)
    check(out[50:60], None, ref, 100, d, dtype)
    assert (out[:50] == 7).all() and (out[60:] == 7).all()
    # sequences that overlap since the offsets fall: twice the same rows
    cu = ints([0, 200] * 150)
    out, lse = S.prompt_attention(q, k, v, cu, want_lse=True)
    torch.cuda.synchronize()
    S.stream_check_device_status()
    check(out, lse, want(q, k, v, [0, 200], [0, 200], True), 200, d, dtype)


@pytest.mark.parametrize("dtype,d", [(BF16, 64), (F32, 64)])
def test_no_tokens(S, dtype, d):
    q, k = torch.zeros(0, 4, d, dtype=dtype, device="cuda"), torch.zeros(0, 2, d, dtype=dtype, device="cuda")
    out, lse = S.prompt_attention(q, k, k, ints([0, 0]), want_lse=True)
    assert out.shape == (0, 4, d) and lse.shape == (4, 0)
    q = torch.randn(5, 4, d, device="cuda").to(dtype)
    out, lse = S.prompt_attention(q, k, k, ints([0, 5]), ints([0, 0]), want_lse=True)
    assert (out == 0).all() and (lse == -float("inf")).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_offsets_beyond_32_bits(S, dtype):
    """Tokens further apart than 2^31 elements in all."""
    n, d = 1100, 64
    q, k, v, cu_q, cu_k = inputs(2, 1, d, [n], [n], dtype)
    base = torch.zeros(n * 2 ** 21 + 64, dtype=dtype, device="cuda")
    far = [base[at:].as_strided((n, h, d), (2 ** 21, 64, 1)) for at, h in ((0, 2), (256, 1), (512, 1))]
    for x, y in zip(far, (q, k, v)):
        x.copy_(y)
    a = S.prompt_attention(q, k, v, ints(cu_q), want_lse=True)
    b = S.prompt_attention(*far, ints(cu_q), want_lse=True)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 256), (F32, 64)])
def test_repeated_on_streams_and_in_a_graph(S, dtype, d):
    q, k, v, cu_q, cu_k = inputs(8, 2, d, [300, 0, 45], [300, 0, 45], dtype)
    cu = ints(cu_q)
    a, la = S.prompt_attention(q, k, v, cu, want_lse=True)
    torch.cuda.synchronize()
    sides = [torch.cuda.Stream() for _ in range(3)]
    outs = [S.prompt_attention(q, k, v, cu, want_lse=True, stream=st) for st in sides for _ in range(2)]  # (at the same time)
    torch.cuda.synchronize()
    for o, lse in outs:
        assert torch.equal(o, a) and torch.equal(lse, la)
    x, lens = q.clone(), cu.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, lse = S.prompt_attention(x, k, v, lens, want_lse=True)
        o2 = S.prompt_attention(o, k, v, lens)
    for other in ([0, 300, 300, 345], [0, 1, 200, 345], [0, 300, 300, 345]):
        lens.copy_(ints(other))
        graph.replay()
        torch.cuda.synchronize()
        e, le = S.prompt_attention(q, k, v, ints(other), want_lse=True)
        assert torch.equal(o, e) and torch.equal(lse, le) and torch.equal(o2, S.prompt_attention(e, k, v, ints(other)))


def test_agrees_with_the_sparse_pass_that_keeps_every_block(S):
    """A mask with as many blocks as there are makes the sparse pass dense."""
    T, d = 1000, 128
    q, k, v = (torch.randn(1, h, T, d, device="cuda").bfloat16() for h in (8, 2, 2))
    mask = S.build_mask(q, k, block_q=64, block_k=64, k_top=16).mask
    sparse = S.sparse_attention(q, k, v, mask, block_q=64, block_k=64)
    dense = S.prompt_attention(*(x[0].transpose(0, 1) for x in (q, k, v)), ints([0, T]))
    w = attention64(*(x[0].transpose(0, 1) for x in (q, k, v)), 0)
    check(dense, None, w, T, d, BF16)
    check(sparse[0].transpose(0, 1), None, w, T, d, BF16)


@pytest.mark.parametrize("keys", [0, 40])
@pytest.mark.parametrize("H,G,d,dtype", [(8, 2, 256, BF16), (8, 2, 128, BF16), (8, 2, 64, BF16), (8, 2, 32, BF16), (7, 1, 16, BF16), (300, 2, 64, BF16),
                                         (8, 2, 128, F32), (8, 1, 256, F32)])
def test_tiles_that_see_no_key_are_zeros_every_time(S, H, G, d, dtype, keys):
    """Thousands of row tiles without any key, of a Q that L2 does not hold: what is stored is never Q, which comes to the place that the output leaves from.
    Without keys at all, and under a causal mask where the last queries alone see one."""
    n = 160 * 2 ** 20 // (H * d * (2 if dtype is BF16 else 4))
    q = torch.full((n, H, d), 3.0, dtype=dtype, device="cuda")
    k, v = (torch.ones(keys, G, d, dtype=dtype, device="cuda") for _ in range(2))
    cu_q, cu_k = ints([0, 1, n // 3, n]), ints([0, 0, 0, keys])
    out, lse = torch.empty_like(q), torch.empty(H, n, device="cuda")
    for _ in range(10):
        out.fill_(5), lse.fill_(5)
        S.prompt_attention(q, k, v, cu_q, cu_k, out=out, lse_out=lse)
        assert not out[:n - keys].any() and (lse[:, :n - keys] == -float("inf")).all()
        assert (out[n - keys:] == 1).all()  # (equal logits: weights of 1, and m (1 / m) is 1 in fp32 up to m = 40)
