"""The operators of a step over drafted token trees refuse bad arguments on the host, before a device is touched; the oracle they are tested
against, on cases small enough to write down."""
import ctypes

import numpy as np
import pytest

import paper_2509_15148_amd as A
from oracle import step_oracle as S
from paper_2509_15148_amd import binding as B

LIB = B._lib
ONE = 4096                                              # a non-NULL, aligned address; never followed


def _desc(**kw):
    base = dict(k_pages=ONE, v_pages=ONE, page_table=ONE, dtype=1, n_pages=4, page_rows=16, n_kv_heads=2, head_dim=128, n_seqs=3, max_pages=8)
    base.update(kw)
    return ctypes.byref(B._PagedDesc(*[base[k] for k, _ in B._PagedDesc._fields_]))


@pytest.mark.parametrize("kw,status", [
    (dict(), 0), (dict(dtype=5), A.ERR_INVALID_ARG), (dict(n_pages=0), A.ERR_INVALID_ARG), (dict(n_kv_heads=0), A.ERR_INVALID_ARG),
    (dict(n_seqs=-1), A.ERR_INVALID_ARG), (dict(max_pages=0), A.ERR_INVALID_ARG), (dict(page_rows=4), A.ERR_SHAPE), (dict(page_rows=48), A.ERR_SHAPE),
    (dict(page_rows=8192), A.ERR_SHAPE), (dict(head_dim=100), A.ERR_SHAPE), (dict(head_dim=264), A.ERR_SHAPE), (dict(head_dim=0), A.ERR_SHAPE),
    (dict(max_pages=1 << 28), A.ERR_SHAPE), (dict(k_pages=0), A.ERR_INVALID_ARG), (dict(page_table=0), A.ERR_INVALID_ARG), (dict(v_pages=8), A.ERR_INVALID_ARG)])
def test_cache_descriptions(kw, status):
    out = ctypes.c_size_t()
    assert LIB.atts_attention_tree_workspace_bytes(_desc(**kw), 8, 10, 4, 100, ctypes.byref(out)) == status
    # no rows: the call ends after its checks
    assert LIB.atts_attention_tree(_desc(**kw), ONE, ONE, ONE, ONE, 0, 8, 4, 100, 1.0, 0.0, 0, ONE, ONE, 1 << 40, None) == status
    assert LIB.atts_rotary_append(_desc(**kw), ONE, 1 << 20, ONE, ONE, ONE, 0, 8, ONE, 1, 16, 0, ONE, None) == status


def test_null_and_misaligned_arguments():
    out = ctypes.c_size_t()
    assert LIB.atts_attention_tree_workspace_bytes(None, 8, 10, 4, 100, ctypes.byref(out)) == A.ERR_INVALID_ARG
    assert LIB.atts_attention_tree_workspace_bytes(_desc(), 8, 10, 4, 100, None) == A.ERR_INVALID_ARG
    assert LIB.atts_attention_tree_workspace_bytes(_desc(), 7, 10, 4, 100, ctypes.byref(out)) == A.ERR_SHAPE
    assert LIB.atts_attention_tree(_desc(), None, ONE, ONE, ONE, 10, 8, 4, 100, 1.0, 0.0, 0, ONE, ONE, 1 << 40, None) == A.ERR_INVALID_ARG
    assert LIB.atts_attention_tree(_desc(), ONE + 2, ONE, ONE, ONE, 10, 8, 4, 100, 1.0, 0.0, 0, ONE, ONE, 1 << 40, None) == A.ERR_INVALID_ARG
    assert LIB.atts_rotary_append(_desc(), ONE, 100, ONE, ONE, ONE, 5, 8, ONE, 1, 16, 0, ONE, None) == A.ERR_INVALID_ARG          # rows overlap
    assert LIB.atts_rotary_append(_desc(), ONE, 1 << 20, ONE, ONE, ONE, 5, 8, None, 1, 16, 0, ONE, None) == A.ERR_INVALID_ARG
    assert LIB.atts_rotary_append(_desc(), ONE, 1 << 20, ONE, ONE, ONE, 5, 8, ONE, 1, 130, 0, ONE, None) == A.ERR_SHAPE
    quant = lambda *a: LIB.atts_gemm_nt_quant(*a[:-1], ONE, 1 << 40, None)
    assert quant(1, ONE, 256, ONE, ONE, None, 64, None, ONE, 0, 8, 256, 0, None) == 0                                             # no rows
    assert quant(2, ONE, 256, ONE, ONE, None, 64, None, ONE, 4, 8, 256, 0, None) == A.ERR_INVALID_ARG
    assert quant(1, ONE, 256, ONE, ONE, None, 48, None, ONE, 4, 8, 96, 0, None) == A.ERR_SHAPE
    assert quant(1, ONE, 256, ONE, ONE, None, 128, None, ONE, 4, 8, 192, 0, None) == A.ERR_SHAPE
    assert quant(1, ONE, 256, ONE, ONE, None, 64, None, ONE, 4, 8, 256, 4, None) == A.ERR_INVALID_ARG
    assert quant(1, ONE, 256, ONE, ONE, None, 64, None, ONE, 4, 8, 256, 2, None) == A.ERR_INVALID_ARG                             # no residual
    assert quant(1, ONE + 8, 256, ONE, ONE, None, 64, None, ONE, 4, 8, 256, 0, None) == A.ERR_INVALID_ARG
    assert quant(1, ONE, 260, ONE, ONE, None, 64, None, ONE, 4, 8, 256, 0, None) == A.ERR_INVALID_ARG
    assert quant(1, ONE, 248, ONE, ONE, None, 64, None, ONE, 4, 8, 256, 0, None) == A.ERR_INVALID_ARG
    assert LIB.atts_quantize_rows(1, None, 8, 256, 64, ONE, ONE, None, None) == A.ERR_INVALID_ARG
    assert LIB.atts_rotary_table(9, 1e4, 64, 1.0, 0.0, 0.0, 0.0, 1.0, 0, 8, ONE, None) == A.ERR_INVALID_ARG
    assert LIB.atts_rotary_table(2, 1e4, 2, 4.0, 0.0, 0.0, 0.0, 1.0, 0, 8, ONE, None) == A.ERR_SHAPE
    assert LIB.atts_rotary_table(0, 1e4, 64, 1.0, 0.0, 0.0, 0.0, 1.0, 0, 0, None, None) == 0
    assert LIB.atts_logits_adjust_workspace_bytes(-1, 10, ctypes.byref(out)) == A.ERR_INVALID_ARG
    assert LIB.atts_logits_adjust_workspace_bytes(3, 0, ctypes.byref(out)) == A.ERR_INVALID_ARG
    adjust = lambda **kw: LIB.atts_logits_adjust(*{**dict(
        dtype=0, logits=ONE, ld=100, off=ONE, n_seqs=2, max_rows=4, params=ONE, hist=None, ho=None, split=None, n_hist=0, ids=None, parents=None, bias=None,
        values=None, bo=None, n_bias=0, mask=None, R=6, V=100, out=ONE, out_ld=100, top=ONE, lse=ONE, ws=ONE, n=1 << 30, stream=None), **kw}.values())
    assert adjust(R=0) == 0 and adjust(n_seqs=0) == 0 and adjust(max_rows=0) == 0
    for kw in (dict(dtype=3), dict(logits=None), dict(off=None), dict(ld=99), dict(out_ld=5), dict(max_rows=257), dict(n_seqs=70000), dict(params=ONE + 4),
               dict(n_hist=4), dict(hist=ONE), dict(ids=ONE), dict(bias=ONE, bo=ONE), dict(n_bias=-1)):
        assert adjust(**kw) == A.ERR_INVALID_ARG, kw
    assert adjust(ws=None) == A.ERR_WORKSPACE and adjust(n=3) == A.ERR_WORKSPACE and adjust(ws=ONE + 16) == A.ERR_WORKSPACE


def test_workspace_never_shrinks_with_the_call():
    size = ctypes.c_size_t()

    def need(nq, R, rows, cached):
        assert LIB.atts_attention_tree_workspace_bytes(_desc(max_pages=1 << 14), nq, R, rows, cached, ctypes.byref(size)) == 0
        return size.value
    for nq in (2, 16):
        last = 0
        for cached in (0, 1, 500, 5000, 9000, 131072, 200000):
            now = max(need(nq, R, rows, cached) for R, rows in ((1, 1), (16, 16), (24, 8)))
            assert now >= last, cached
            last = now
        for R in (1, 2, 3, 7, 16, 40, 300, 2000):
            assert need(nq, R, min(R, 7), 70000) <= need(nq, R + 1, min(R + 1, 7), 70000)


# ---- the oracle itself ----------------------------------------------------------------------------------------------

def test_oracle_quantization():
    codes = np.array([[0x21, 0xF0]], dtype=np.uint8)                    # 1, 2, 0, 15
    w = S.dequantize(codes, np.array([[0.5, 2.0]]), np.array([[1, 3]]))
    assert w.tolist() == [[0.0, 0.5, -6.0, 24.0]]
    assert S.dequantize(codes, np.array([[0.5, 2.0]]), None).tolist() == [[-3.5, -3.0, -16.0, 14.0]]
    q, scale, zero = S.quantize(np.array([[-1.0, 0.0, 0.6, 2.0]]), 4, False, lambda s: s)
    assert zero.tolist() == [[5]] and q.tolist() == [[0, 5, 8, 15]] and np.allclose(scale, 0.2)
    q, scale, zero = S.quantize(np.array([[0.0, 0.0], [8.0, -7.0]]), 2, True, lambda s: s)
    assert q.tolist() == [[8, 8], [15, 2]] and zero.tolist() == [[8], [8]] and scale[0, 0] == 0


def test_oracle_rotation():
    quarter = np.array([[[0.0, 1.0]]])                                  # cos, sin of a quarter turn
    x = np.array([[[1.0, 2.0, 3.0]]])
    assert S.rotate(x, quarter, True).tolist() == [[[-2.0, 1.0, 3.0]]]
    assert S.rotate(x[..., :2], quarter, False).tolist() == [[[-2.0, 1.0]]]
    f = S.rotary_frequencies(100.0, 4)
    assert np.allclose(f, [1.0, 0.1]) and np.allclose(S.rotary_frequencies(100.0, 4, "linear", 2.0), f / 2)
    assert np.allclose(S.rotary_frequencies(100.0, 4, "stretched", 4.0), [1.0, 1.0 / 40])          # 100 x 4^2
    turns = 1000 * f / (2 * np.pi)
    parts = S.rotary_frequencies(100.0, 4, "by_parts", 2.0, 1000.0, turns[1] - 1, turns[1] + 1)
    assert np.allclose(parts, [1.0, 0.075])                             # beyond high: as it is; half way: between f and f / 2


def test_oracle_tree_attention():
    assert S.path([-1, 0, 0, 5, -3, 2], 5) == [5, 2, 0] and S.path([-1, 0, 0, 5, -3], 3) == [3]
    k = np.zeros((4, 1, 2))
    v = np.array([[[1.0, 0]], [[3.0, 0]], [[5.0, 0]], [[np.nan, 0]]])
    out = S.tree_attention(np.ones((3, 1, 2)), k, v, [-1, -1, 1], 1, 1.0)       # rows 1, 2, 3; row 1 sees 1.0, 5.0
    assert out[0, 0, 0] == 2.0 and out[1, 0, 0] == 3.0 and np.isnan(out[2, 0, 0])
    assert S.tree_attention(np.ones((2, 1, 2)), k, v, [-1, -1], 1, 1.0, window=1)[:, 0, 0].tolist() == [3.0, 5.0]


def test_oracle_logits():
    x, top = S.adjust(np.array([2.0, -2.0, 1.0, 8.0]), (2.0, 0.5, 0.25, 0.5), [3], [1, 1, 9], {0: 1.0}, np.array([1, 1, 1, 0], bool))
    assert x.tolist() == [6.0, -10.5, 2.0, -np.inf] and top == 0
    assert S.adjust(np.array([1.0, np.nan]), None, [], [], {}, np.array([0, 1], bool))[1] == -1
    assert S.log_sum_exp(np.array([0.0, 0.0])) == np.log(2) and S.log_sum_exp(np.array([-np.inf])) == -np.inf
