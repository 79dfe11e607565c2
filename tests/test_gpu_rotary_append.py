"""Rotary table and rotary append against the 64-bit oracle: layouts, part of the head, page sizes, ragged sequences, rows and pages out of range."""
import numpy as np
import pytest
import torch

import paper_2509_15148_amd as A
from oracle import step_oracle as S
from step_util import DTYPES, UNIT, Paged, host, i32, offsets
from util import announce

pytestmark = pytest.mark.gpu
SCALINGS = {"plain": A.ROTARY_PLAIN, "linear": A.ROTARY_LINEAR, "stretched": A.ROTARY_STRETCHED, "by_parts": A.ROTARY_BY_PARTS}


@pytest.mark.parametrize("scaling", list(SCALINGS))
@pytest.mark.parametrize("rot,first", [(4, 0), (64, 100), (128, 131000), (256, 1000000)])
def test_table(scaling, rot, first):
    kw = dict(plain={}, linear=dict(factor=4.0), stretched=dict(factor=8.0), by_parts=dict(factor=8.0, original=4096.0, low=1.0, high=32.0))[scaling]
    table = torch.full((300, rot // 2, 2), float("nan"), device="cuda")
    announce("rotary table", scaling, rot, first)
    A.atts_rotary_table(table, 10000.0, SCALINGS[scaling], magnitude=1.25, first=first, **kw)
    ang = np.arange(first, first + 300)[:, None] * S.rotary_frequencies(10000.0, rot, scaling, **kw)
    want = 1.25 * np.stack([np.cos(ang), np.sin(ang)], axis=-1)
    # angles up to 1e6 in 64 bits, their frequencies good to a few units of 2^-53: 1e6 2^-50 = 1e-9; then one rounding to 32 bits
    assert np.abs(table.cpu().numpy() - want).max() <= 1.25 * 2.0 ** -24 + 2e-9


def _case(lens, cached, nq, nkv, hd, rot, page, dtype, interleaved, seed, stride_pad=0):
    rng = np.random.default_rng(seed)
    R = sum(lens)
    p = Paged(rng, [c + n for c, n in zip(cached, lens)], nkv, page, hd, dtype, fill=7.0)
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(R, (nq + 2 * nkv) * hd, generator=g).to(dtype)
    room = torch.full((max(R, 1), x.shape[1] + stride_pad), float("nan"), dtype=dtype, device="cuda")
    room[:R, :x.shape[1]] = x.cuda()
    n_pos = max([c + n for c, n in zip(cached, lens)] + [1])
    table = torch.randn(n_pos, rot // 2, 2, generator=g)
    positions = rng.integers(0, n_pos, R)
    q = torch.full((R, nq * hd), float("nan"), dtype=dtype, device="cuda")
    before_k, before_v = p.k.clone(), p.v.clone()
    A.atts_rotary_append(p.cache, room[:R, :x.shape[1]], i32(positions), i32(cached), i32(offsets(lens)), table.cuda(),
                         A.ROTARY_INTERLEAVED if interleaved else A.ROTARY_HALF, q)
    y = host(x).reshape(R, nq + 2 * nkv, hd).astype(np.float64)
    turned = S.rotate(y[:, :nq + nkv], table.numpy()[positions], interleaved)
    # two products and their sum in 32 bits, at most 3 units of 2^-24 of |a c| + |b s| <= the largest entry of the table times |a| + |b|; one rounding
    big = float(table.abs().max()) if rot else 1.0
    tol = 3 * 2.0 ** -24 * big * 2 * float(np.abs(y).max()) if R else 0.0
    close = lambda got, want: (np.abs(got - want) <= tol + UNIT[dtype] * np.abs(want) * 1.01).all()
    assert close(host(q), turned[:, :nq].reshape(R, -1))
    seen_k, seen_v = torch.zeros(p.k.shape[0], page, dtype=torch.bool), torch.zeros(p.k.shape[0], page, dtype=torch.bool)
    k, v = host(p.k), host(p.v)
    r = 0
    for s, n in enumerate(lens):
        for i in range(n):
            pg, slot = p.table_np[s, (cached[s] + i) // page], (cached[s] + i) % page
            assert close(k[pg, :, slot], turned[r, nq:]) and np.array_equal(v[pg, :, :, slot], y[r, nq + nkv:].astype(np.float32)), (s, i)
            seen_k[int(pg), slot] = True
            r += 1
    others = ~seen_k.cuda()
    assert torch.equal(p.k.transpose(1, 2)[others], before_k.transpose(1, 2)[others])          # nothing else was written
    assert torch.equal(p.v.permute(0, 3, 1, 2)[others], before_v.permute(0, 3, 1, 2)[others])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("lens,cached,nq,nkv,hd,rot,page", [
    ([1], [0], 1, 1, 8, 8, 8), ([1, 1, 1], [0, 15, 16], 4, 2, 128, 128, 16), ([5, 0, 17, 1], [3, 9, 30, 100], 7, 1, 64, 32, 16),
    ([70], [0], 4, 4, 32, 32, 32), ([3, 40], [61, 7], 2, 2, 96, 48, 64), ([33, 2], [5, 0], 3, 3, 72, 6, 8), ([9], [2], 6, 2, 256, 256, 16),
    ([20, 20], [1, 2], 0, 2, 40, 0, 16), ([200, 1, 0], [100, 3, 5], 8, 8, 128, 64, 256), ([600], [13], 2, 1, 128, 128, 16)])
def test_append(dtype, interleaved, lens, cached, nq, nkv, hd, rot, page):
    announce("append", dtype, interleaved, lens, cached, nq, nkv, hd, rot, page)
    _case(lens, cached, nq, nkv, hd, rot, page, dtype, interleaved, seed=hd + page)


def test_strided_rows():
    for dtype, pad in ((torch.bfloat16, 8), (torch.bfloat16, 3), (torch.float32, 1)):
        announce("append strided", dtype, pad)
        _case([5, 12], [3, 30], 4, 2, 64, 64, 16, dtype, False, seed=pad, stride_pad=pad)


def test_many_sequences():
    rng = np.random.default_rng(3)
    lens, cached = [int(n) for n in rng.integers(0, 4, 300)], [int(c) for c in rng.integers(0, 40, 300)]
    announce("append 300 sequences")
    _case(lens, cached, 2, 1, 32, 32, 16, torch.bfloat16, False, seed=9)


def test_values_out_of_range_do_not_fault_or_store():
    """Rows past a sequence's pages, pages that do not exist, positions outside the table, rows no sequence owns."""
    hd, page = 32, 16
    k = torch.full((2, 1, page, hd), 7.0, device="cuda")
    v = torch.full((2, 1, hd, page), 7.0, device="cuda")
    cache = A.PagedCache(k, v, i32([[0, 5], [-3, 1]]))
    R = 8
    qkv = torch.randn(R, 3 * hd, device="cuda")
    table = torch.zeros(4, hd // 2, 2, device="cuda")
    table[..., 0] = 1.0                                            # no rotation
    q = torch.full((R, hd), float("nan"), device="cuda")
    announce("append out of range")
    # sequence 0: tokens 15 (stored), 16 (page 5 of 2), sequence 1: tokens 15 (page -3), 16 (page 1, stored), ..., 18 (page 1)
    A.atts_rotary_append(cache, qkv, i32([0, 9, -4, 3, 0, 0, 0, 0]), i32([15, 15]), i32([0, 2, 6]), table, A.ROTARY_HALF, q)
    assert torch.equal(q, qkv[:, :hd])
    kw = torch.full_like(k, 7.0)
    kw[0, 0, 15], kw[1, 0, 0:3] = qkv[0, hd:2 * hd], qkv[3:6, hd:2 * hd]
    assert torch.equal(k, kw)
    vw = torch.full_like(v, 7.0)
    vw[0, 0, :, 15], vw[1, 0, :, 0:3] = qkv[0, 2 * hd:], qkv[3:6, 2 * hd:].t()
    assert torch.equal(v, vw)
    A.atts_rotary_append(cache, qkv, i32([0] * 8), i32([31, 32]), i32([0, 2, 6]), table, A.ROTARY_HALF, q)       # the end of the table, and behind it
    vw, kw = v.clone(), k.clone()
    A.atts_rotary_append(cache, qkv, i32([0] * 8), i32([2 ** 31 - 1, -5]), i32([0, 2, 6]), table, A.ROTARY_HALF, q)
    torch.cuda.synchronize()
    kw[0, 0, :1], vw[0, 0, :, :1] = k[0, 0, :1], v[0, 0, :, :1]
    assert torch.equal(k, kw) and torch.equal(v, vw)


def test_refusals():
    hd = 32
    k, v = torch.zeros(2, 1, 16, hd, device="cuda"), torch.zeros(2, 1, hd, 16, device="cuda")
    cache = A.PagedCache(k, v, i32([[0, 1]]))
    qkv, q, table = torch.zeros(3, 4 * hd, device="cuda"), torch.zeros(3, 2 * hd, device="cuda"), torch.zeros(8, hd // 2, 2, device="cuda")
    pos, cached, off = i32([0, 1, 2]), i32([0]), i32([0, 3])

    def refused(code, f, *a):
        with pytest.raises(A.AttsError) as e:
            f(*a)
        assert e.value.code == code
    bad = lambda code, *a: refused(code, A.atts_rotary_append, *a)
    bad(A.ERR_INVALID_ARG, cache, qkv, pos, cached, off, table, 2, q)
    bad(A.ERR_INVALID_ARG, cache, qkv.bfloat16(), pos, cached, off, table, 0, q)
    bad(A.ERR_INVALID_ARG, cache, qkv, pos[:2], cached, off, table, 0, q)
    bad(A.ERR_INVALID_ARG, cache, qkv, pos, cached, off[:1], table, 0, q)
    bad(A.ERR_INVALID_ARG, cache, qkv, pos, cached, off, table, 0, q[:, :hd])
    bad(A.ERR_INVALID_ARG, cache, qkv[:, :hd], pos, cached, off, table, 0, q)
    bad(A.ERR_SHAPE, cache, qkv, pos, cached, off, torch.zeros(8, hd, 2, device="cuda"), 0, q)           # more pairs than the head has
    bad(A.ERR_INVALID_ARG, cache, qkv, pos, cached, off, table[:0], 0, q)
    refused(A.ERR_INVALID_ARG, A.PagedCache, k, v.transpose(2, 3).contiguous(), i32([[0, 1]]))
    odd = A.PagedCache(torch.zeros(2, 1, 24, hd, device="cuda"), torch.zeros(2, 1, hd, 24, device="cuda"), i32([[0, 1]]))
    bad(A.ERR_SHAPE, odd, qkv, pos, cached, off, table, 0, q)
    refused(A.ERR_INVALID_ARG, A.atts_rotary_table, table, -1.0)
    refused(A.ERR_INVALID_ARG, A.atts_rotary_table, table, 1e4, A.ROTARY_LINEAR, 0.0)
    refused(A.ERR_INVALID_ARG, A.atts_rotary_table, table, 1e4, A.ROTARY_BY_PARTS, 2.0, 0.0)
    A.atts_rotary_append(cache, qkv[:0], pos[:0], cached, i32([0, 0]), table, 0, q[:0])
