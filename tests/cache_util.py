"""Paged caches for the GPU tests: rows in scattered pages of several memory orders, everything that no row owns is NaN."""
import numpy as np
import torch

from gpu_util import to_host
from oracle import cache as oc

DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def normal(seed, *shape, dtype="bf16", std=1.0):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * std).to(DT[dtype]).cuda()


def pool(pages, page, hk, d, dtype, order="page,row,head"):
    """Two pools of NaN, [pages, page, hk, d] each."""
    dt = DT[dtype]
    new = lambda *shape: torch.full(shape, float("nan"), dtype=dt, device="cuda")
    if order == "page,row,head":
        return new(pages, page, hk, d), new(pages, page, hk, d)
    if order == "page,head,row":
        return new(pages, hk, page, d).transpose(1, 2), new(pages, hk, page, d).transpose(1, 2)
    if order == "pages of both":
        t = new(pages, 2, page, hk, d)
        return t[:, 0], t[:, 1]
    t = new(pages, page, 2 * hk, d)                              # rows of both
    return t[:, :, :hk], t[:, :, hk:]


class Batch:
    """A cache with `lens` random rows per sequence, of which the last `new` are the call's tokens."""

    def __init__(self, seed, new, lens, hq, hk, d, page, dtype="bf16", order="page,row,head", pad=0, spare=2, max_new=None, path=0):
        import paper_2503_21817_b200 as sk
        self.new, self.lens, self.hq, self.hk, self.d, self.page, self.dtype = list(new), list(lens), hq, hk, d, page, dtype
        need = [-(-n // page) for n in lens]
        total = sum(need) + spare
        rng = np.random.default_rng(seed)
        perm = rng.permutation(total)
        self.table = np.full((len(lens), max(need + [1])), -1, dtype=np.int32)
        at = 0
        for i, n in enumerate(need):
            self.table[i, :n] = perm[at:at + n]
            at += n
        self.free = perm[at:]
        self.k, self.v = pool(total, page, hk, d, dtype, order)
        self.keys, self.values = [], []
        for i, n in enumerate(lens):
            rows = [normal(seed + 10 * i + j, n, hk, d, dtype=dtype) for j in (1, 2)]
            j = torch.arange(n, device="cuda")
            pages = torch.from_numpy(self.table[i]).cuda().long()[j // page]
            self.k[pages, j % page], self.v[pages, j % page] = rows
            self.keys.append(to_host(rows[0]))
            self.values.append(to_host(rows[1]))
        self.cu = [0] + [int(c) for c in np.cumsum(new)]
        self.q = normal(seed + 3, self.cu[-1] + pad, hq, d, dtype=dtype, std=1.3)
        dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
        self.d_table, self.d_cu, self.d_lens = torch.from_numpy(self.table).cuda(), dev(self.cu), dev(self.lens)
        self.cache = sk.PagedCache(self.k, self.v, self.d_table, self.d_cu, self.d_lens, max(new) if max_new is None else max_new, path=path)
        self.scale = d ** -0.5

    def want(self, scale=None):
        return oc.attention(to_host(self.q)[:self.cu[-1]], self.keys, self.values, self.cu, self.lens, scale or self.scale, self.dtype)


def within(got, want, bound, what):
    got = to_host(got)
    assert got.shape == want.shape, what
    both = np.isneginf(want)
    assert np.array_equal(np.isneginf(got), both), what
    got, want = np.where(both, 0.0, got), np.where(both, 0.0, want)
    assert np.isfinite(got).all(), f"{what}: non-finite values"
    worst = np.max(np.abs(got - want) / np.maximum(bound, 1e-300)) if got.size else 0.0
    assert worst <= 1.0, f"{what}: an element is {worst:.3f} times its bound away"
