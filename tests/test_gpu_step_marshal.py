"""Both ways of a step's operators, native marshalling and the general one, make the same call; what the native one does not take is worded by the
general one."""
import numpy as np
import pytest
import torch

import paper_2509_15148_amd as A
from paper_2509_15148_amd import binding as B
from step_util import Paged, i32, tree
from util import announce, ws


def test_what_is_not_plain_is_left_to_the_general_way():
    m, other, host, cache = B._marshal, B._marshal.OTHER, torch.zeros(4, 4), B._PagedDesc()
    for f, n in ((m.gemm_nt_quant, 8), (m.rotary_append, 8), (m.attention_tree, 12), (m.logits_adjust, 17)):
        for args in ([], [None] * n, [host] * n, [B.ctypes.addressof(cache)] + [host] * (n - 1), [0] + [None] * (n - 1), ["x"] * n):
            assert f(*args) == other
        assert f(*[torch.empty(4, 4, device="meta")] * n) == other


@pytest.mark.gpu
def test_both_ways_make_the_same_call(monkeypatch):
    announce("step marshal both ways")
    rng, g = np.random.default_rng(1), torch.Generator(device="cuda").manual_seed(2)
    dt, nq, nkv, hd, lens, cached = torch.bfloat16, 4, 2, 64, [5, 0, 3], [100, 4, 0]
    R, V = sum(lens), 3000
    r = lambda *shape: torch.randn(*shape, device="cuda", generator=g)
    x, codes = r(R, 256).to(dt), torch.randint(0, 256, (512, 128), dtype=torch.uint8, device="cuda", generator=g)
    scales, zeros = r(512, 4).abs().to(dt), torch.randint(0, 16, (512, 4), dtype=torch.uint8, device="cuda", generator=g)
    p = Paged(rng, [c + n for c, n in zip(cached, lens)], nkv, 16, hd, dt, fill=0.5)
    parents, offsets, length = i32([t for n in lens for t in tree(rng, n)]), i32([0, 5, 5, 8]), i32(cached)
    rotary, logits = r(128, hd // 2, 2), r(R, V)
    params, history = torch.rand(3, 4, device="cuda", generator=g) + 0.5, i32(rng.integers(0, V, 90))
    calls = {}
    for way in ("native", "general"):
        used = []
        for name in ("gemm_nt_quant", "rotary_append", "attention_tree", "logits_adjust"):
            native = getattr(B._marshal, name)
            monkeypatch.setattr(B._marshal, name, (lambda *a, f=native: used.append(f(*a)) or used[-1]) if way == "native" else lambda *a: B._marshal.OTHER)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            qkv = torch.empty(R, (nq + 2 * nkv) * hd, dtype=dt, device="cuda")
            A.atts_gemm_nt_quant(x, codes, scales, zeros, qkv)
            up, res = torch.empty(R, 256, dtype=dt, device="cuda"), r(R, 512) * 0 + 1.0
            A.atts_gemm_nt_quant(x, codes, scales, None, up, A.EPILOGUE_SWIGLU)
            A.atts_gemm_nt_quant(x, codes, scales, zeros, res, A.EPILOGUE_RESIDUAL, res)
            wide = torch.empty(40, 512, dtype=dt, device="cuda")
            A.atts_gemm_nt_quant(x.repeat(5, 1), codes, scales, zeros, wide)
            q, out = torch.empty(R, nq * hd, dtype=dt, device="cuda"), torch.empty(R, nq * hd, dtype=dt, device="cuda")
            A.atts_rotary_append(p.cache, qkv, i32([100, 101, 102, 103, 104, 0, 1, 2]), length, offsets, rotary, A.ROTARY_INTERLEAVED, q)
            A.atts_attention_tree(p.cache, q, parents, length, offsets, 5, 100, out, ws(A.atts_attention_tree_workspace_bytes(p.cache, nq, R, 5, 100)), None, 20.0, 50)
            adjusted, top, lse = torch.empty_like(logits), i32([0] * R), torch.empty(R, device="cuda")
            A.atts_logits_adjust(logits, offsets, params, history, i32([0, 30, 60, 90]), i32([10, 0, 30]), i32(rng.integers(0, 9, R) * 0 + 7), parents, None, None, None,
                                 None, adjusted, top, lse, ws(A.atts_logits_adjust_workspace_bytes(R, V)), max_rows=5)
        torch.cuda.synchronize()
        assert way == "general" or used.count(0) == 7             # every call went through in native code
        calls[way] = [t.cpu() for t in (qkv, up, res, wide, q, out, p.k, p.v, adjusted, top, lse)]
        monkeypatch.undo()
    assert all(torch.equal(a, b) for a, b in zip(calls["native"], calls["general"]))


@pytest.mark.gpu
def test_errors_are_the_general_way_s():
    announce("step marshal errors")
    x = torch.zeros(2, 64, dtype=torch.bfloat16, device="cuda")
    codes, scales, out = torch.zeros(8, 32, dtype=torch.uint8, device="cuda"), torch.zeros(8, 2, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 8, dtype=torch.bfloat16, device="cuda")
    for call, text in ((lambda: A.atts_gemm_nt_quant(x, codes, scales, None, out.cpu()), "device tensor"),
                       (lambda: A.atts_gemm_nt_quant(x, codes, scales, None, out[:, :4]), "shape mismatch"),
                       (lambda: A.atts_gemm_nt_quant(x, codes[:, ::2], scales, None, out), "shape mismatch"),
                       (lambda: A.atts_gemm_nt_quant(x.double(), codes, scales, None, out), "unsupported dtype|must have dtype"),
                       (lambda: A.atts_gemm_nt_quant(x, codes, scales, None, out, 9), "epilogue")):
        with pytest.raises(A.AttsError, match=text) as e:
            call()
        assert e.value.code == A.ERR_INVALID_ARG
