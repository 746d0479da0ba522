"""A paged cache on the GPU beside its copy for the oracle."""
import numpy as np
import torch

from paper_2605_29707_amd import binding as bd

DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def dev(x, dtype=None):
    return torch.as_tensor(x, device=DEV, dtype=dtype)


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


class Pages:
    """Caches of `layers` layers for sequences of the given lengths; room: slots that each one's pages hold beyond its
    length.  Pages are in random order, unused table entries name no page, unused rows hold NaN."""

    def __init__(self, lens, page=16, nkv=2, dh=64, dtype="bf16", order="slot", layers=1, room=0, weights=False, seed=0,
                 stale="nan", spare=3):
        rng = np.random.RandomState(seed)
        self.page, self.nkv, self.dh, self.dtype, self.layers, self.lens = page, nkv, dh, DT[dtype], layers, np.asarray(lens, np.int32)
        need = [-(-(n + room) // page) for n in lens]
        self.pages = sum(need) + spare
        perm = rng.permutation(self.pages).astype(np.int32)
        self.table = np.full((len(lens), max(need + [1]) + 2), -1, np.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = perm[at:at + n]
            at += n
        self.free = perm[at:]
        a, b = (page, nkv) if order == "slot" else (nkv, page)
        g = torch.Generator().manual_seed(seed)
        fill = lambda: torch.randn(layers, self.pages, a, b, dh, generator=g).to(self.dtype)  # noqa: E731
        k, v = fill(), fill()
        if order == "head":
            k, v = k.transpose(2, 3), v.transpose(2, 3)
        if stale == "nan":
            used = torch.zeros(self.pages, page, dtype=torch.bool)
            for s, n in enumerate(lens):
                for i in range(n):
                    used[self.table[s, i // page], i % page] = True
            k[:, ~used] = float("nan")
            v[:, ~used] = float("nan")
        self.k, self.v = k.to(DEV), v.to(DEV)
        assert self.k.stride() == k.stride()
        self.w = torch.rand(layers, self.pages, nkv, page, generator=g).to(DEV) if weights else None
        self.cache = bd.PagedCache(self.k, self.v, i32(self.table), weights=self.w)

    def copies(self):
        w = None if self.w is None else self.w.cpu().numpy().copy()
        return self.k.float().cpu().numpy(), self.v.float().cpu().numpy(), w

    def workspace(self, n):
        return torch.zeros(n, dtype=torch.uint8, device=DEV)


def starts_of(news):
    return np.concatenate([[0], np.cumsum(news)]).astype(np.int32)


def half_step(dtype):
    return torch.finfo(dtype).eps / 2
