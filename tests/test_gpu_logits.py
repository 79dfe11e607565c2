"""Logits under penalties, biases, temperature and masks: bit for bit what the steps give in 32 bits, rounded one by one; log-sum-exp against 64 bits."""
import numpy as np
import pytest
import torch

import paper_2509_15148_amd as A
from oracle import step_oracle as S
from step_util import DTYPES, host, i32, offsets, tree
from util import announce, dirty_ws

pytestmark = pytest.mark.gpu


class Case:
    def __init__(self, V, lens, hist, dtype, bias=0, mask=False, paths=True, seed=0, params=True):
        rng = np.random.default_rng(seed)
        self.V, self.lens, self.dtype, self.R, n = V, lens, dtype, sum(lens), len(lens)
        self.logits = torch.from_numpy(rng.standard_normal((self.R, V)).astype(np.float32) * 3).to(dtype)
        ids = lambda m: (V * rng.random(m) ** 3).astype(np.int32)
        self.hist = [ids(h) for h in hist]
        self.split = [int(rng.integers(0, h + 1)) for h in hist]
        self.params = np.stack([rng.uniform(1, 1.5, n), rng.uniform(-0.2, 0.6, n), rng.uniform(0, 0.6, n), rng.uniform(0.5, 1.5, n)], axis=1).astype(np.float32) \
            if params else None
        self.parents = [tree(rng, m) for m in lens]
        self.tree_ids = [ids(m) for m in lens]
        self.paths = paths
        self.bias = [list(zip(rng.integers(0, V, bias).tolist(), (rng.standard_normal(bias) * 4).astype(np.float32).tolist())) for _ in lens]
        self.mask = None
        if mask:
            self.mask = rng.random((self.R, -(-V // 32) * 32)) < rng.choice([0.02, 0.5, 0.98], (self.R, 1))

    def words(self):
        return i32(np.packbits(self.mask, axis=1, bitorder="little").view("<u4").astype(np.int64).astype(np.uint32).view(np.int32))

    def expected(self):
        rows, top, r = [], [], 0
        for s, n in enumerate(self.lens):
            for i in range(n):
                own = self.tree_ids[s][S.path(self.parents[s], i)].tolist() if self.paths else []
                x, best = S.adjust(host(self.logits[r]), None if self.params is None else self.params[s], self.hist[s][:self.split[s]].tolist(),
                                   self.hist[s][self.split[s]:].tolist() + own, dict(self.bias[s]), None if self.mask is None else self.mask[r, :self.V])
                rows.append(x)
                top.append(best)
                r += 1
        return rows, top

    def run(self, in_place=False, decide=True, pad=0):
        d = self.logits.cuda()
        if pad:
            wide = torch.full((self.R, self.V + pad), 5.0, dtype=self.dtype, device="cuda")
            wide[:, :self.V] = d
            d = wide[:, :self.V]
        out = d if in_place else torch.full((self.R, self.V), 9.0, dtype=self.dtype, device="cuda")
        top = torch.full((self.R,), -9, dtype=torch.int32, device="cuda") if decide else None
        lse = torch.full((self.R,), 9.0, device="cuda") if decide else None
        space = dirty_ws(A.atts_logits_adjust_workspace_bytes(self.R, self.V)) if decide else None
        cat = lambda parts, dt: torch.tensor(np.concatenate(parts) if parts else [], dtype=dt, device="cuda")
        bias = any(self.bias)
        A.atts_logits_adjust(
            d, i32(offsets(self.lens)), None if self.params is None else torch.from_numpy(self.params).cuda(),
            cat(self.hist, torch.int32), i32(offsets([len(h) for h in self.hist])), i32(self.split),
            cat(self.tree_ids, torch.int32) if self.paths else None, cat([np.array(p) for p in self.parents], torch.int32) if self.paths else None,
            i32([t for b in self.bias for t, _ in b]) if bias else None,
            torch.tensor([v for b in self.bias for _, v in b], dtype=torch.float32, device="cuda") if bias else None,
            i32(offsets([len(b) for b in self.bias])) if bias else None, self.words() if self.mask is not None else None, out, top, lse, space,
            max_rows=max(max(self.lens), 1))
        return out, top, lse

    def check(self, got):
        out, top, lse = got
        rows, best = self.expected()
        for r, x in enumerate(rows):
            want = torch.from_numpy(x).to(self.dtype)
            assert torch.equal(torch.nan_to_num(out[r].cpu(), nan=1e30), torch.nan_to_num(want, nan=1e30)), r
            if top is not None:
                assert int(top[r]) == best[r], r
                want_lse, z = S.log_sum_exp(x), float(lse[r])
                # terms good to 2^-22 relative (exp of up to 40 off by 40 2^-24), their sum in pieces: 1e-5 in the logarithm; its own rounding
                assert z == want_lse or (np.isnan(z) and np.isnan(want_lse)) or abs(z - want_lse) <= 1e-5 + 2.0 ** -22 * abs(want_lse), (r, z, want_lse)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V,lens,hist,bias,mask", [
    (1, [1], [0], 0, False), (7, [3], [20], 3, True), (31, [1, 0, 2], [5, 5, 0], 0, True), (1024, [5, 1], [300, 0], 10, False),
    (4096, [2], [1000], 5, True), (4097, [1, 1, 1], [10, 100, 3], 0, True), (33000, [4, 16], [5000, 1], 300, True), (152064, [1], [2000], 20, False),
    (128256, [3, 1], [30000, 4], 0, True), (50001, [40], [700], 8, False)])
def test_rules(dtype, V, lens, hist, bias, mask):
    announce("logits", dtype, V, lens, hist, bias, mask)
    c = Case(V, lens, hist, dtype, bias, mask, seed=V)
    c.check(c.run())


@pytest.mark.parametrize("dtype", DTYPES)
def test_parts_left_out(dtype):
    for kw in (dict(paths=False), dict(params=False, mask=True), dict(params=False, bias=4), dict(params=False)):
        announce("logits parts", dtype, kw)
        c = Case(9000, [3, 2], [50, 0], dtype, seed=1, **kw)
        c.check(c.run())
    c = Case(9000, [3, 2], [0, 0], dtype, seed=2)
    c.check(c.run(decide=False))
    c.check(c.run())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pad", [0, 1, 8])
def test_in_place_and_strided(dtype, pad):
    c = Case(5003, [4, 3], [100, 7], dtype, bias=5, mask=True, seed=3)
    announce("logits in place", dtype, pad)
    got = c.run(in_place=True, pad=pad)
    c.check(got)
    if pad:
        assert bool((got[0]._base[:, c.V:] == 5.0).all())


@pytest.mark.parametrize("dtype", DTYPES)
def test_empty_rows_ties_and_special_values(dtype):
    c = Case(6000, [4, 4], [30, 30], dtype, mask=True, params=False, paths=False, seed=4)
    c.mask[:] = True
    c.mask[0] = False                                      # nothing is allowed
    c.mask[1, :], c.mask[1, 5999] = False, True            # the very last token alone
    c.logits[2, [100, 4500, 99]] = 50.0                    # ties: the lowest index
    c.logits[3, 7] = float("nan")
    c.logits[4] = -float("inf")                            # allowed, but nothing above -inf
    c.logits[5, 4321] = float("inf")
    c.logits[6, 4321], c.logits[6, 5], c.mask[6, 5] = -float("inf"), float("nan"), False      # a masked NaN never shows
    c.logits[7] = torch.finfo(dtype).min
    announce("logits special", dtype)
    out, top, lse = c.run()
    c.check((out, top, lse))
    assert top.tolist()[:3] == [-1, 5999, 99] and int(top[4]) == -1 and int(top[5]) == 4321 and int(top[7]) == 0
    assert float(lse[0]) == -np.inf and np.isnan(float(lse[3])) and float(lse[5]) == np.inf and np.isfinite(float(lse[6]))


def test_long_paths_and_ids_out_of_range():
    c = Case(3000, [256, 5], [40, 40], torch.float32, bias=4, seed=5)
    c.parents = [list(range(-1, 255)), [3, -7, 1, 2 ** 31 - 1, 0]]
    c.tree_ids[0][::3], c.tree_ids[1][2] = 17, -1
    c.hist[0][5], c.hist[0][30], c.hist[1][0] = 3000, -2 ** 31, 2 ** 31 - 1
    c.bias[0][1] = (-1, 100.0)
    announce("logits long paths")
    c.check(c.run())


def test_last_of_several_biases_counts():
    c = Case(5000, [2], [10], torch.float32, bias=600, seed=6)
    c.bias[0] = [(t % 40 * 100, v) for t, v in c.bias[0]]
    announce("logits repeated biases")
    c.check(c.run())


def test_offsets_out_of_range_and_rows_of_nobody():
    c = Case(5000, [3], [10], torch.float32, seed=7)
    d, out = c.logits.cuda(), torch.full((3, 5000), 9.0, device="cuda")
    top, space = torch.full((3,), -9, dtype=torch.int32, device="cuda"), dirty_ws(A.atts_logits_adjust_workspace_bytes(3, 5000))
    announce("logits offsets")
    A.atts_logits_adjust(d, i32([0, 2]), torch.tensor([[1.0, 0.0, 0.0, 1.0]], device="cuda"), i32(c.hist[0]), i32([-5, 2 ** 31 - 1]), i32([2 ** 31 - 1]), None, None,
                         None, None, None, None, out, top, None, space)
    assert torch.equal(out[:2], d[:2]) and bool((out[2] == 9.0).all()) and int(top[2]) == -9
    assert top[:2].tolist() == d[:2].argmax(dim=1).tolist()


def test_same_bits_again():
    c = Case(152064, [5, 9], [3000, 3000], torch.float32, bias=30, mask=True, seed=8)
    announce("logits twice")
    one, two = c.run(), c.run()
    assert all(torch.equal(a, b) for a, b in zip(one, two))


def test_refusals():
    c = Case(100, [2], [5], torch.float32, seed=9)
    d, off, par = c.logits.cuda(), i32([0, 2]), torch.from_numpy(c.params).cuda()
    out, top, space = torch.empty_like(d), i32([0, 0]), dirty_ws(A.atts_logits_adjust_workspace_bytes(2, 100))
    none = [None] * 6

    def refused(code, *a, **k):
        with pytest.raises(A.AttsError) as e:
            A.atts_logits_adjust(*a, **k)
        assert e.value.code == code
    h = [i32([1, 2]), i32([0, 2]), None]
    refused(A.ERR_INVALID_ARG, d, off, par[:, :3].contiguous(), *h, None, None, None, None, None, None, out, top, None, space)
    refused(A.ERR_INVALID_ARG, d, off, par, h[0], None, None, None, None, None, None, None, None, out, top, None, space)
    refused(A.ERR_INVALID_ARG, d, off, par, *h, i32([1, 1]), None, None, None, None, None, out, top, None, space)
    refused(A.ERR_INVALID_ARG, d, off, par, *h, None, None, i32([1]), None, None, None, out, top, None, space)
    refused(A.ERR_INVALID_ARG, d, off, par, *h, None, None, None, None, None, i32([[1, 1]]), out, top, None, space)
    refused(A.ERR_INVALID_ARG, d, off, par, *h, None, None, None, None, None, None, out.bfloat16(), top, None, space)
    refused(A.ERR_INVALID_ARG, d, off, par, *h, None, None, None, None, None, None, out[:1], top, None, space)
    refused(A.ERR_INVALID_ARG, d, off, par, *h, None, None, None, None, None, None, out, top, None, space, max_rows=300)
    refused(A.ERR_WORKSPACE, d, off, par, *h, None, None, None, None, None, None, out, top, None, None)
    refused(A.ERR_WORKSPACE, d, off, par, *h, None, None, None, None, None, None, out, None, torch.empty(2, device="cuda"), space[:16])
    A.atts_logits_adjust(d[:0], i32([0, 0]), par, *h, None, None, None, None, None, None, out[:0], top[:0], None, space)
