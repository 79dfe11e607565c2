"""Inputs of the tests of a step over drafted token trees: paged caches with pages in no order, trees, types."""
import numpy as np
import torch

NP = {torch.float32: np.float32, torch.bfloat16: np.float32}
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}      # half a unit in the last of 24 and of 8 significant bits
DTYPES = [torch.float32, torch.bfloat16]


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def host(t):
    return t.detach().float().cpu().numpy()


def tree(rng, n, kind="branches"):
    """Parents of n rows."""
    if kind == "chain":
        return list(range(-1, n - 1))
    if kind == "flat":
        return [-1] * n
    return [i - 1 if rng.random() < 0.5 else int(rng.integers(-1, i)) if i else -1 for i in range(n)]


def offsets(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


class Paged:
    """A cache for sequences of `total` tokens each; whatever no sequence owns is `fill`."""

    def __init__(self, rng, total, nkv, page, hd, dtype, fill=float("nan"), spare=2):
        import paper_2509_15148_amd as A
        need = [-(-t // page) for t in total]
        n = sum(need) + spare
        self.order = rng.permutation(n)
        self.width = max(max(need), 1)
        table = np.full((len(total), self.width), -7, dtype=np.int32)          # entries no token needs are not valid pages
        at = 0
        for s, m in enumerate(need):
            table[s, :m] = self.order[at:at + m]
            at += m
        self.table_np, self.page, self.nkv, self.hd, self.dtype = table, page, nkv, hd, dtype
        self.k = torch.full((n, nkv, page, hd), fill, dtype=dtype, device="cuda")
        self.v = torch.full((n, nkv, hd, page), fill, dtype=dtype, device="cuda")
        self.table = i32(table)
        self.cache = A.PagedCache(self.k, self.v, self.table)

    def put(self, s, first, k, v):
        """k, v [tokens, nkv, hd] (torch, cpu) into tokens first .. of sequence s"""
        for j in range(k.shape[0]):
            page, slot = self.table_np[s, (first + j) // self.page], (first + j) % self.page
            self.k[int(page), :, slot] = k[j].to(self.dtype).cuda()
            self.v[int(page), :, :, slot] = v[j].to(self.dtype).cuda()

    def fill_sequence(self, s, k, v):
        """the same for whole sequences, page by page"""
        m = k.shape[0]
        for i in range(-(-m // self.page)):
            a, b = i * self.page, min((i + 1) * self.page, m)
            page = int(self.table_np[s, i])
            self.k[page, :, :b - a] = k[a:b].to(self.dtype).cuda().transpose(0, 1)
            self.v[page, :, :, :b - a] = v[a:b].to(self.dtype).cuda().permute(1, 2, 0)
