"""Dense attention and the paged cache in 64 bits and in plain Python, for the tests of the kernels.

How far a kernel may be off, element by element, is counted from its arithmetic (u = 2^-24, half a step of fp32):
  logits      d products added in fp32, scaled: off by at most (d + 2) u M, M the largest scale * sum_c |q_c k_c| of the row
  weights     2^x off by 2^-22 relative, x by the above and a rounding of |x| (x a difference of logits: at most 2 M log2 e,
              rounded twice): all weights relative to their sum by twice that
  sums        n + 2 terms in fp32, any order: (n + 2) u relative, in the numerator and in the denominator
  bf16        weights rounded for the product: 2^-8 of each, so 2^-8 A, A = sum_j p_j |v_j|; the output: 2^-8 |o|
"""
import math

import torch

U = 2.0 ** -24


def attention64(q, k, v, first, scale=None):
    """q [n, H, d], k and v [m, G, d]; query i sees keys j <= first + i (all if first is None). In 64 bits: output, logarithm of
    the sums [H, n], sum_j p_j |v_j|, and the largest scale * sum_c |q_c k_c| of a row [n, H]."""
    n, H, d = q.shape
    m, G = k.shape[:2]
    scale = 1 / math.sqrt(d) if scale is None else scale
    out, mag = torch.zeros(n, H, d, dtype=torch.float64, device=q.device), torch.zeros(n, H, d, dtype=torch.float64, device=q.device)
    lse, top = torch.full((H, n), -math.inf, dtype=torch.float64, device=q.device), torch.zeros(n, H, dtype=torch.float64, device=q.device)
    if n and m:
        seen = torch.ones(n, m, dtype=torch.bool, device=q.device)
        if first is not None:
            seen = torch.arange(m, device=q.device)[None] <= torch.arange(n, device=q.device)[:, None] + first
        for h in range(H):
            a, b, w = q[:, h].double(), k[:, h * G // H].double(), v[:, h * G // H].double()
            s = (a @ b.T * scale).masked_fill(~seen, -math.inf)
            ls = torch.logsumexp(s, 1)
            p = torch.exp(s - torch.where(ls > -math.inf, ls, 0.0)[:, None])
            out[:, h], mag[:, h], lse[h] = p @ w, p @ w.abs(), ls
            top[:, h] = (a.abs() @ b.abs().T * scale).masked_fill(~seen, 0.0).amax(1)
    return out, lse, mag, top


def check(got, lse, want, n_keys, d, dtype, what=""):
    """Outputs of a kernel against attention64's."""
    out, ls, mag, top = want
    logit = (d + 2) * U * top
    weight = 2 * (logit + 2 ** -22 + 8 * U * top) + 2 * (n_keys + 2) * U
    rel = 2.0 ** -8 if dtype is torch.bfloat16 else U
    bound = rel * out.abs() + mag * weight[..., None] * (1 + 2.0 ** -6) + 1e-30
    if dtype is torch.bfloat16:
        bound = bound + 2.0 ** -8 * mag * (1 + 2.0 ** -6)
    off = (got.double() - out).abs()
    assert torch.isfinite(got.float()).all(), what
    assert (off <= bound).all(), (what, float((off / bound).max()))
    if lse is not None:
        empty = ls == -math.inf
        assert torch.equal(lse == -math.inf, empty), what
        far = (lse.double() - ls).abs()[~empty]
        most = (logit.T + weight.T + 4 * U * ls.abs() + 2 ** -21)[~empty]
        assert (far <= most).all(), (what, float((far / most).max()))


def offsets(lens):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return at


def ints(x, device="cuda"):
    return torch.tensor(x, dtype=torch.int32, device=device)


class Ledger:
    """The ledger in plain Python: what the calls leave, and their info."""

    def __init__(self, n_slots, n_pages, page, max_pages):
        self.page, self.max_pages = page, max_pages
        self.table = [[-1] * max_pages for _ in range(n_slots)]
        self.len, self.count = [0] * n_slots, [0] * n_pages

    def free_pages(self):
        return [p for p, c in enumerate(self.count) if c == 0]

    def pages(self, n):
        return -(-n // self.page)

    def reserve(self, new):
        free = self.free_pages()
        bad = sum(n < 0 or self.pages(m + n) > self.max_pages for m, n in zip(self.len, new))
        need = sum(self.pages(m + n) - self.pages(m) for m, n in zip(self.len, new) if n >= 0 and self.pages(m + n) <= self.max_pages)
        if bad or need > len(free):
            return [0, need, len(free), bad]
        at = iter(free)
        for s, n in enumerate(new):
            for j in range(self.pages(self.len[s]), self.pages(self.len[s] + n)):
                self.table[s][j] = next(at)
                self.count[self.table[s][j]] = 1
            self.len[s] += n
        return [1, need, len(free) - need, 0]

    def fork(self, parent):
        n = len(parent)
        free = self.free_pages()
        child = [s for s in range(n) if parent[s] >= 0]
        bad = sum(parent[s] >= n or parent[parent[s]] >= 0 or self.len[s] != 0 for s in child)
        need = sum(self.len[parent[s]] % self.page != 0 for s in child
                   if parent[s] < n and parent[parent[s]] < 0 and self.len[s] == 0)
        if bad or need > len(free):
            return [[-1, -1]] * n, [0, need, len(free), bad]
        pairs, at = [], iter(free)
        for s in child:
            p = parent[s]
            for j in range(self.pages(self.len[p])):
                x = self.table[p][j]
                if (j + 1) * self.page > self.len[p]:
                    pairs.append([x, next(at)])
                    x = pairs[-1][1]
                self.table[s][j] = x
                self.count[x] += 1
            self.len[s] = self.len[p]
        return pairs + [[-1, -1]] * (n - len(pairs)), [1, need, len(free) - need, 0]

    def free(self, done):
        before = len(self.free_pages())
        for s, x in enumerate(done):
            if x:
                for y in self.table[s][:self.pages(self.len[s])]:
                    self.count[y] -= 1
                self.table[s], self.len[s] = [-1] * self.max_pages, 0
        after = len(self.free_pages())
        return [1, after - before, after, 0]

    def compact(self):
        n_pages = len(self.count)
        free = self.free_pages()
        used = n_pages - len(free)
        moves = [list(x) for x in zip([p for p in range(used, n_pages) if self.count[p]], [p for p in free if p < used])]
        to = {a: b for a, b in moves}
        self.table = [[to.get(x, x) for x in row] for row in self.table]
        for a, b in moves:
            self.count[b], self.count[a] = self.count[a], 0
        return moves + [[-1, -1]] * (n_pages // 2 - len(moves)), [1, len(moves), len(free), 0]

    def tensors(self, device="cuda"):
        return ints(self.table, device).view(len(self.len), self.max_pages), ints(self.len, device), ints(self.count, device)

    def same(self, cache):
        table, length, count = self.tensors(cache.device)
        return torch.equal(cache.page_table, table) and torch.equal(cache.seq_len, length) and torch.equal(cache.ref_count, count)


def filled_cache(S, lens, page, G, d, dtype, *, n_layers=1, spare=3, order="lpthd", seed=0, max_pages=None, garbage=float("nan")):
    """A cache whose slots hold `lens` tokens on pages in a shuffled order, and the keys and values of each slot and layer. What no
    token is in holds `garbage`. order: how the dimensions (layer, page, token, head, d) lie in memory."""
    gen = torch.Generator("cuda").manual_seed(seed)
    need = [-(-n // page) for n in lens]
    n_pages = sum(need) + spare
    max_pages = max_pages or max(need + [1]) + 1
    sizes = dict(l=n_layers, p=n_pages, t=page, h=G, d=d)
    perm = [order.index(x) for x in "lpthd"]
    k, v = (torch.full([sizes[x] for x in order], garbage, dtype=dtype, device="cuda").permute(perm) for _ in range(2))
    pages = torch.randperm(n_pages, generator=gen, device="cuda").tolist()
    led = Ledger(len(lens), n_pages, page, max_pages)
    rows = []
    for s, n in enumerate(lens):
        kk, vv = (torch.randn(n_layers, n, G, d, generator=gen, device="cuda").to(dtype) for _ in range(2))
        rows.append((kk, vv))
        led.len[s] = n
        for j in range(need[s]):
            x = led.table[s][j] = pages.pop()
            led.count[x] = 1
            m = min(page, n - j * page)
            k[:, x, :m], v[:, x, :m] = kk[:, j * page:j * page + m], vv[:, j * page:j * page + m]
    return S.PagedCache(k, v, *led.tensors()), rows, led
