"""Attention under any mask, and the paged cache in 8 bits, in 64 bits and in plain Python, for the tests of the kernels.

Tolerances as in ``serve_helpers``. Over a cache in 8 bits the arithmetic differs in this (the numbers of the cache are given, and exact):
  q           times a power of two in fp16, its largest element in [2^14, 2^15): a bf16 number is exact but for what lies below 2^-25, 2^-39 of the largest;
              of an fp32 one two fp16 numbers leave 2^-22
  weights     bf16: rounded to fp16, 2^-11 of each; fp32: two fp16 numbers, 2^-22. Both: what lies below 2^-25, the largest weight times its value's
              scale being in (2^13, 2^15]: off by 2^-38 of that product, times 448 scales at most
"""
import math

import torch

from serve_helpers import U, Ledger

E4M3 = torch.float8_e4m3fn


def seen_by(n, m, window, sinks, device="cuda"):
    """n queries, the last at the last of m keys."""
    p, j = torch.arange(m - n, m, device=device)[:, None], torch.arange(m, device=device)[None]
    return (j <= p) & ((j > p - window) | (j < sinks)) if window else j <= p


def masked64(q, k, v, seen, scale=None):
    """As serve_helpers.attention64, under a mask [n, m]."""
    n, H, d = q.shape
    m, G = k.shape[:2]
    scale = 1 / math.sqrt(d) if scale is None else scale
    out, mag = (torch.zeros(n, H, d, dtype=torch.float64, device=q.device) for _ in range(2))
    lse, top = torch.full((H, n), -math.inf, dtype=torch.float64, device=q.device), torch.zeros(n, H, dtype=torch.float64, device=q.device)
    if n and m:
        for h in range(H):
            a, b, w = q[:, h].double(), k[:, h * G // H].double(), v[:, h * G // H].double()
            s = (a @ b.T * scale).masked_fill(~seen, -math.inf)
            ls = torch.logsumexp(s, 1)
            p = torch.exp(s - torch.where(ls > -math.inf, ls, 0.0)[:, None])
            out[:, h], mag[:, h], lse[h] = p @ w, p @ w.abs(), ls
            top[:, h] = (a.abs() @ b.abs().T * scale).masked_fill(~seen, 0.0).amax(1)
    return out, lse, mag, top


def check8(got, lse, q, k, v, v_scale, scale, dtype, what=""):
    """One query [H, d] against its keys [m, G, d] in 64 bits; v_scale [m, G]: what a value's e4m3 numbers are multiplied by."""
    H, d = q.shape
    m, G = k.shape[:2]
    scale = 1 / math.sqrt(d) if scale is None else scale
    if m == 0:
        assert (got == 0).all() and (lse == -math.inf).all(), what
        return
    a = q.double()
    b, w, z = (x.double().repeat_interleave(H // G, 1) for x in (k, v, v_scale))  # of each query head
    s = torch.einsum("hd,mhd->hm", a, b) * scale
    ls = torch.logsumexp(s, 1)
    p = torch.exp(s - ls[:, None])
    out, mag = torch.einsum("hm,mhd->hd", p, w), torch.einsum("hm,mhd->hd", p, w.abs())
    top = torch.einsum("hd,mhd->hm", a.abs(), b.abs()).amax(1) * scale
    bf16 = dtype is torch.bfloat16
    logit = (d + 2) * U * top + scale * a.abs().amax(1) * b.abs().sum(2).amax(0) * 2.0 ** -39 + (0 if bf16 else 2.0 ** -22 * top)
    weight = 2 * (logit + 2 ** -22 + 8 * U * top) + 2 * (m + 2) * U
    each = weight * (1 + 2.0 ** -6) + (2.0 ** -11 if bf16 else 2.0 ** -22)
    cut = m * 2.0 ** -38 * 448 * (p * z.T).amax(1)
    bound = (2.0 ** -8 if bf16 else U) * out.abs() + mag * each[:, None] * (1 + 2.0 ** -6) + cut[:, None] + 1e-30
    off = (got.double() - out).abs()
    assert torch.isfinite(got.float()).all(), what
    assert (off <= bound).all(), (what, float((off / bound).max()))
    far = (lse.double() - ls).abs()
    assert (far <= logit + weight + 4 * U * ls.abs() + 2 ** -21).all(), (what, float(far.max()))


def scale_of(top):
    """The smallest 2^e, -90 <= e <= 120, with top <= 448 2^e; of whole tensors, in 64 bits."""
    e = torch.full_like(top, -90.0, dtype=torch.float64)
    for x in range(-89, 121):
        e = torch.where(top.double() > 448 * 2.0 ** (x - 1), float(x), e)
    return torch.exp2(e)


def rounded8(x):
    """The nearest e4m3 numbers, ties to even, of numbers up to 448; in 64 bits."""
    e = torch.frexp(x.abs().clamp(min=2.0 ** -6)).exponent - 4
    unit = torch.exp2(e.double())
    return torch.round(x / unit) * unit


class Slots8:
    """What the slots of a cache in 8 bits hold: of each a list of layers of {K, V}: [values [n, G, d], scales [blocks, G]] in 64 bits."""

    def __init__(self, n_slots, n_layers, block, G, d, device="cuda"):
        self.block = block
        zero = lambda: [torch.zeros(0, G, d, dtype=torch.float64, device=device), torch.zeros(0, G, dtype=torch.float64, device=device)]  # noqa: E731
        self.held = [[[zero(), zero()] for _ in range(n_layers)] for _ in range(n_slots)]

    def write(self, s, layer, kv, rows):
        x, scales = self.held[s][layer][kv]
        n, m = x.shape[0], rows.shape[0]
        if m == 0:
            return
        x, scales, block = torch.cat([x, rows.double()]), scales.clone(), self.block
        for b in range(n // block, -(-(n + m) // block)):
            lo, hi = b * block, min(n + m, (b + 1) * block)
            z = scale_of(x[max(lo, n):hi].abs().amax((0, 2)))
            if lo < n:
                z = torch.maximum(z, scales[b])
                scales[b] = z
            else:
                scales = torch.cat([scales, z[None]])
            x[lo:hi] = rounded8(x[lo:hi] / z[None, :, None]) * z[None, :, None]
        self.held[s][layer][kv] = [x, scales]

    def scales_by_token(self, s, layer, kv):
        x, scales = self.held[s][layer][kv]
        return scales.repeat_interleave(self.block, 0)[:x.shape[0]]


def empty_cache8(S, n_slots, page, block, G, d, dtype, need, *, n_layers=1, spare=3, max_pages=8, order="lpthd", scale_order="lpbh"):
    """All slots empty, what no token is in being NaN. need: pages."""
    n_pages = need + spare
    sizes = dict(l=n_layers, p=n_pages, t=page, h=G, d=d, b=page // block)
    k, v = (torch.full([sizes[x] for x in order], 127, dtype=torch.uint8, device="cuda").view(E4M3).permute([order.index(x) for x in "lpthd"]) for _ in range(2))
    ks, vs = (torch.full([sizes[x] for x in scale_order], float("nan"), device="cuda").permute([scale_order.index(x) for x in "lpbh"]) for _ in range(2))
    led = Ledger(n_slots, n_pages, page, max_pages)
    return S.PagedCache8(k, v, ks, vs, *led.tensors(), dtype=dtype), led


def filled_cache8(S, lens, page, block, G, d, dtype, *, n_layers=1, seed=0, size=None, **kw):
    """A cache whose slots hold `lens` tokens on pages in a shuffled order, put there without the library; and what they hold. size: of the
    blocks' values, [blocks of a slot at most], or None."""
    gen = torch.Generator("cuda").manual_seed(seed)
    need = [-(-n // page) for n in lens]
    cache, led = empty_cache8(S, len(lens), page, block, G, d, dtype, sum(need), n_layers=n_layers, max_pages=max(need + [1]) + 1, **kw)
    pages = torch.randperm(cache.n_pages, generator=gen, device="cuda").tolist()
    held = Slots8(len(lens), n_layers, block, G, d)
    for s, n in enumerate(lens):
        led.len[s] = n
        for j in range(need[s]):
            led.table[s][j] = pages.pop()
            led.count[led.table[s][j]] = 1
        for layer in range(n_layers):
            for kv in range(2):
                x = torch.randn(n, G, d, generator=gen, device="cuda")
                if size is not None:
                    x *= size[torch.arange(n, device="cuda") // block][:, None, None]
                nb = -(-n // block)
                grouped = torch.zeros(nb * block, G, d, dtype=torch.float64, device="cuda")
                grouped[:n] = x
                grouped = grouped.view(nb, block, G, d)
                z = scale_of(grouped.abs().amax((1, 3)))
                y = rounded8(grouped / z[:, None, :, None])
                held.held[s][layer][kv] = [(y * z[:, None, :, None]).view(-1, G, d)[:n], z]
                raw = y.float().to(E4M3).view(torch.uint8).view(-1, G, d)[:n]
                to, to_scale = (cache.k, cache.k_scale) if kv == 0 else (cache.v, cache.v_scale)
                to = to.view(torch.uint8)
                for j in range(need[s]):
                    m, x_page = min(page, n - j * page), led.table[s][j]
                    to[layer, x_page, :m] = raw[j * page:j * page + m]
                    bpp = page // block
                    part = z[j * bpp:(j + 1) * bpp].float()
                    to_scale[layer, x_page, :part.shape[0]] = part
    cache.page_table.copy_(led.tensors()[0]), cache.seq_len.copy_(led.tensors()[1]), cache.ref_count.copy_(led.tensors()[2])
    return cache, held, led
