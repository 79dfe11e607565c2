"""Attention of drafted token trees over a paged cache against the 64-bit oracle.  Whatever no row may see is NaN: slots behind a sequence's end,
pages of nobody, and, where a test says so, the keys and values of other branches."""
import numpy as np
import pytest
import torch

import paper_2509_15148_amd as A
from oracle import step_oracle as S
from step_util import DTYPES, UNIT, Paged, host, i32, offsets, tree
from util import announce, dirty_ws

pytestmark = pytest.mark.gpu


def _inputs(lens, cached, nq, nkv, hd, page, dtype, kind, seed, qscale=1.0):
    rng, g = np.random.default_rng(seed), torch.Generator().manual_seed(seed)
    p = Paged(rng, [c + n for c, n in zip(cached, lens)], nkv, page, hd, dtype)
    kv = []
    for s, (c, n) in enumerate(zip(cached, lens)):
        k, v = (torch.randn(c + n, nkv, hd, generator=g).to(dtype) for _ in range(2))
        p.fill_sequence(s, k, v)
        kv.append((host(k), host(v)))
    q = (torch.randn(sum(lens), nq * hd, generator=g) * qscale).to(dtype)
    return p, kv, q, [tree(rng, n, kind) for n in lens]


def _run(p, q, parents, cached, lens, stream=None, max_rows=None, max_cached=None, **kw):
    out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
    nq = q.shape[1] // p.hd
    max_rows, max_cached = max_rows or max(max(lens), 1), max_cached or max(cached)
    space = dirty_ws(A.atts_attention_tree_workspace_bytes(p.cache, nq, q.shape[0], max_rows, max_cached))
    A.atts_attention_tree(p.cache, q.cuda(), i32([x for t in parents for x in t]), i32(cached), i32(offsets(lens)), max_rows, max_cached, out, space, **kw)
    return out


def _tolerance(q, k, v, hd, dtype, scale, softcap):
    """A score's sum of hd products in 32 bits is off by at most 2 sqrt(hd) units of 2^-24 of its terms' sizes (a cap adds the tanh's and the
    quotient's roundings, 8 units of the cap); exp adds 4 units.  A probability's relative error counts twice, itself and in the sum, times the largest
    value; 16 bits: every probability rounded to 2^-8 once more."""
    sizes = scale * np.abs(q).max() * np.abs(k).sum(axis=-1).max()
    dz = 2.0 ** -24 * (2 * hd ** 0.5 * sizes + 8 * softcap + 4 + 2 * sizes)
    return np.abs(v).max() * (2 * dz + 2.0 ** -22 + (2.0 ** -8 if dtype == torch.bfloat16 else 0.0))


def _check(got, q, kv, parents, cached, lens, nq, hd, dtype, scale=None, softcap=0.0, window=0):
    scale, r = hd ** -0.5 if scale is None else scale, 0
    got = host(got).reshape(-1, nq, hd)
    qn = host(q).reshape(-1, nq, hd)
    for s, n in enumerate(lens):
        if n:
            k, v = kv[s]
            ref = S.tree_attention(qn[r:r + n], k, v, parents[s], cached[s], scale, softcap, window)
            err = np.abs(got[r:r + n] - ref)
            tol = _tolerance(qn[r:r + n], np.nan_to_num(k), np.nan_to_num(v), hd, dtype, scale, softcap) + UNIT[dtype] * 1.01 * np.abs(ref)
            assert (err <= tol).all(), (s, float(err.max()), float(tol.max()))
        r += n


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lens,cached,nq,nkv,hd,page,kind", [
    ([1], [0], 1, 1, 8, 8, "chain"), ([1], [1], 4, 4, 32, 8, "chain"), ([1, 1], [17, 300], 8, 2, 64, 16, "chain"),
    ([7], [100], 7, 1, 128, 16, "branches"), ([16, 0, 3], [5, 40, 127], 8, 8, 128, 32, "branches"), ([33], [63], 4, 2, 96, 64, "branches"),
    ([64], [65], 16, 2, 64, 16, "flat"), ([20, 1, 40], [0, 700, 31], 10, 2, 128, 16, "branches"), ([5], [513], 6, 3, 72, 8, "branches"),
    ([12], [200], 4, 1, 256, 16, "branches"), ([100], [50], 4, 2, 128, 16, "branches"), ([256], [33], 2, 1, 64, 16, "branches"),
    ([256], [0], 8, 1, 128, 128, "chain"), ([9, 9, 9, 9], [1000, 3, 64, 128], 28, 4, 128, 16, "branches"), ([3], [2500], 12, 1, 40, 256, "branches")])
def test_trees(dtype, lens, cached, nq, nkv, hd, page, kind):
    announce("tree", dtype, lens, cached, nq, nkv, hd, page, kind)
    p, kv, q, parents = _inputs(lens, cached, nq, nkv, hd, page, dtype, kind, seed=hd + page + sum(lens))
    _check(_run(p, q, parents, cached, lens), q, kv, parents, cached, lens, nq, hd, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("softcap,window,scale", [(5.0, 0, None), (0.0, 1, None), (0.0, 2, 0.3), (30.0, 64, None), (0.0, 100, None), (2.0, 33, 1.0), (0.0, 5000, -0.1)])
def test_caps_and_windows(dtype, softcap, window, scale):
    lens, cached, nq, nkv, hd = [24, 1, 5], [150, 64, 0], 8, 2, 64
    announce("tree cap window", dtype, softcap, window, scale)
    p, kv, q, parents = _inputs(lens, cached, nq, nkv, hd, 16, dtype, "branches", seed=17, qscale=2.0)
    got = _run(p, q, parents, cached, lens, softcap=softcap, window=window, scale=scale)
    s = hd ** -0.5 if scale is None else scale
    _check(got, q, kv, parents, cached, lens, nq, hd, dtype, s, softcap, window) if s > 0 else \
        _check(got, -q.float(), kv, parents, cached, lens, nq, hd, dtype, -s, softcap, window)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cached,page,n", [(20000, 64, 3), (9001, 16, 1), (4097, 32, 40)])
def test_long_contexts(dtype, cached, page, n):
    announce("tree long", dtype, cached, page, n)
    nq, nkv, hd = 4, 2, 128
    p, kv, q, parents = _inputs([n], [cached], nq, nkv, hd, page, dtype, "branches", seed=n)
    _check(_run(p, q, parents, [cached], [n]), q, kv, parents, [cached], [n], nq, hd, dtype)
    got = _run(p, q, parents, [cached], [n], window=777)
    _check(got, q, kv, parents, [cached], [n], nq, hd, dtype, window=777)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("where", ["key", "value"])
def test_another_branch_never_shows(dtype, bad, where):
    """Two branches; one's key or value is bad: its descendants show it, the other branch is what it would be without."""
    lens, cached, nq, nkv, hd = [10], [40], 8, 2, 64
    p, kv, q, _ = _inputs(lens, cached, nq, nkv, hd, 16, dtype, "chain", seed=3)
    parents = [[-1, 0, 1, 2, 3, -1, 5, 6, 7, 8]]
    announce("tree bad branch", dtype, bad, where)
    page, slot = int(p.table_np[0, 42 // 16]), 42 % 16
    if where == "key":
        p.k[page, :, slot] = bad
    else:
        p.v[page, :, :, slot] = bad
    got = _run(p, q, parents, cached, lens)
    assert bool(torch.isfinite(got[:2].float()).all()) and bool(torch.isfinite(got[5:].float()).all())
    if where == "value":
        assert not bool(torch.isfinite(got[2:5].float()).any())
    else:                                            # a key of infinities: scores of +inf, -inf or NaN; those of NaN and +inf show
        assert bool(torch.isnan(got[2:5].float()).any())
    keep = [0, 1, 5, 6, 7, 8, 9]
    clean = host(got).reshape(10, nq, hd)
    ref = S.tree_attention(host(q).reshape(10, nq, hd), *kv[0], parents[0], 40, hd ** -0.5)
    tol = _tolerance(host(q), *kv[0], hd, dtype, hd ** -0.5, 0.0) + UNIT[dtype] * 1.01 * np.abs(ref[keep])
    assert (np.abs(clean[keep] - ref[keep]) <= tol).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_bad_value_behind_the_window_never_shows(dtype):
    lens, cached, nq, nkv, hd = [4], [300], 4, 2, 128
    p, kv, q, parents = _inputs(lens, cached, nq, nkv, hd, 16, dtype, "chain", seed=8)
    for j in (0, 100, 203):                          # rows at positions 300 .. 303 with a window of 100 see 201 .. on
        page, slot = int(p.table_np[0, j // 16]), j % 16
        p.k[page, :, slot], p.v[page, :, :, slot] = float("nan"), float("nan")
    announce("tree bad window", dtype)
    got = host(_run(p, q, parents, cached, lens, window=100)).reshape(4, nq, hd)
    bad = np.isnan(got).reshape(4, -1)
    assert bad[:3].all() and not bad[3].any()        # token 203 is out of sight for the last row alone
    k, v = (np.nan_to_num(x) for x in kv[0])
    ref = S.tree_attention(host(q).reshape(4, nq, hd), k, v, parents[0], 300, hd ** -0.5, window=100)
    assert (np.abs(got[3] - ref[3]) <= _tolerance(host(q), k, v, hd, dtype, hd ** -0.5, 0.0) + UNIT[dtype] * 1.01 * np.abs(ref[3])).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_large_scores(dtype):
    """Scores of several hundred, one key far ahead: nothing overflows, and the running maximum moves late and early."""
    lens, cached, nq, nkv, hd = [3], [900], 2, 1, 64
    p, kv, q, parents = _inputs(lens, cached, nq, nkv, hd, 16, dtype, "chain", seed=21, qscale=30.0)
    announce("tree large scores", dtype)
    _check(_run(p, q, parents, cached, lens), q, kv, parents, cached, lens, nq, hd, dtype)


def test_values_out_of_range_do_not_fault():
    """Parents that are no earlier row, pages that do not exist (read as page 0), more cached tokens and rows than announced."""
    lens, cached, nq, nkv, hd, page = [6, 4], [30, 20], 4, 2, 64, 16
    p, kv, q, parents = _inputs(lens, cached, nq, nkv, hd, page, torch.bfloat16, "chain", seed=2)
    wild = [[5, -9, 1, 3, 2 ** 31 - 1, 4], [0, 1, -2 ** 31, 2]]
    announce("tree out of range")
    _check(_run(p, q, wild, cached, lens), q, kv, wild, cached, lens, nq, hd, torch.bfloat16)
    p.table[0, 1], p.table[1, 0] = 2 ** 31 - 1, -1
    p.k[0], p.v[0] = 0.0, 1.0
    assert bool(torch.isfinite(_run(p, q, parents, cached, lens).float()).all())
    few = _run(p, q, parents, cached, lens, max_rows=3, max_cached=10)
    assert bool(torch.isnan(few[3:6].float()).all()) and bool(torch.isnan(few[9:].float()).all())          # rows past max_rows are left alone
    wide = _run(p, q, parents, [2 ** 31 - 1, -3], lens, max_cached=1000)
    torch.cuda.synchronize()
    assert wide.shape == q.shape


@pytest.mark.parametrize("dtype", DTYPES)
def test_same_bits_again_and_on_another_stream(dtype):
    lens, cached, nq, nkv, hd = [20, 7], [5000, 64], 8, 2, 128
    p, kv, q, parents = _inputs(lens, cached, nq, nkv, hd, 16, dtype, "branches", seed=6)
    announce("tree twice", dtype)
    one = _run(p, q, parents, cached, lens)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        two = _run(p, q, parents, cached, lens)
    side.synchronize()
    assert torch.equal(one, two)


def test_refusals():
    p, kv, q, parents = _inputs([4], [10], 4, 2, 64, 16, torch.float32, "chain", seed=1)
    par, cached, off, out, qd = i32(parents[0]), i32([10]), i32([0, 4]), torch.empty(4, 256, device="cuda"), q.cuda()
    need = A.atts_attention_tree_workspace_bytes(p.cache, 4, 4, 4, 10)
    space = dirty_ws(need)

    def refused(code, *a, **k):
        with pytest.raises(A.AttsError) as e:
            A.atts_attention_tree(*a, **k)
        assert e.value.code == code
    refused(A.ERR_INVALID_ARG, p.cache, qd, par, cached, off, 257, 10, out, space)
    refused(A.ERR_INVALID_ARG, p.cache, qd, par, cached, off, 4, -1, out, space)
    refused(A.ERR_INVALID_ARG, p.cache, qd.bfloat16(), par, cached, off, 4, 10, out, space)
    refused(A.ERR_INVALID_ARG, p.cache, qd, par[:3], cached, off, 4, 10, out, space)
    refused(A.ERR_INVALID_ARG, p.cache, qd, par, cached, off, 4, 10, out[:, :128], space)
    refused(A.ERR_INVALID_ARG, p.cache, qd, par, cached, off, 4, 10, out, space, softcap=-1.0)
    refused(A.ERR_INVALID_ARG, p.cache, qd, par, cached, off, 4, 10, out, space, softcap=float("nan"))
    refused(A.ERR_INVALID_ARG, p.cache, qd, par, cached, off, 4, 10, out, space, scale=float("inf"))
    refused(A.ERR_INVALID_ARG, p.cache, qd, par, cached, off, 4, 10, out, space, window=-1)
    refused(A.ERR_SHAPE, p.cache, qd[:, :192].contiguous(), par, cached, off, 4, 10, out[:, :192].contiguous(), space)
    big = A.atts_attention_tree_workspace_bytes(p.cache, 4, 4, 4, 100000)
    if big:
        refused(A.ERR_WORKSPACE, p.cache, qd, par, cached, off, 4, 100000, out, None)
        refused(A.ERR_WORKSPACE, p.cache, qd, par, cached, off, 4, 100000, out, dirty_ws(big)[:big - 1])
    A.atts_attention_tree(p.cache, qd[:0], par[:0], cached, i32([0, 0]), 4, 10, out[:0], space)
