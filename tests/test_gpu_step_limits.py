"""The operators of a step where their kernels change over: histories longer than 16 bits count, many sequences, histories of many slices, every shape of
the 4-bit products' tiles and splits, heads of 256, caches past 2^31 elements; captured in a graph and replayed."""
import numpy as np
import pytest
import torch

import paper_2509_15148_amd as A
from step_util import DTYPES, UNIT, Paged, host, i32, offsets, tree
from test_gpu_logits import Case
from test_gpu_quant import _check as check_product, _inputs as product_inputs, _run as run_product
from test_gpu_rotary_append import _case as append_case
from test_gpu_tree import _check as check_tree, _inputs as tree_inputs, _run as run_tree
from util import announce, dirty_ws, ws

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [65279, 65280, 70001])
def test_histories_around_16_bits(n):
    """One token most of the time, so that its count passes 16 bits where the history does; the path counts on top."""
    announce("long history", n)
    c = Case(300, [40], [n], torch.float32, seed=n)
    c.hist[0][:] = np.where(np.arange(n) % 100 < 99, 7, c.hist[0])
    for split in (0, n, n // 3):
        c.split, c.parents, c.tree_ids = [split], [list(range(-1, 39))], [np.full(40, 7, dtype=np.int32)]
        c.params[:] = [[1.3, 1e-5, 0.5, 0.8]]
        c.check(c.run())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V,n_seqs,bias", [(5003, 600, 0), (4096, 1030, 3), (33000, 120, 0), (70000, 60, 0), (40001, 110, 5)])
def test_many_sequences_of_logits(dtype, V, n_seqs, bias):
    announce("logits many", dtype, V, n_seqs, bias)
    rng = np.random.default_rng(V)
    lens = [int(n) for n in rng.integers(0, 2, n_seqs)]
    c = Case(V, lens, [int(h) for h in rng.integers(0, 60, n_seqs)], dtype, bias=bias, mask=True, seed=n_seqs)
    c.check(c.run())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V,bias", [(130000, 0), (130001, 0), (130000, 3), (130001, 3)])
def test_many_long_histories(dtype, V, bias):
    announce("logits long histories", dtype, V, bias)
    c = Case(V, [1 + s % 2 for s in range(33)], [9000 - 10 * s for s in range(33)], dtype, bias=bias, mask=V % 2 == 0, seed=V)
    c.check(c.run())


@pytest.mark.parametrize("M", [17, 32, 33, 70])
@pytest.mark.parametrize("N,K,group,epilogue", [(64, 4096, 32, "store"), (200, 2048, 128, "swiglu"), (1100, 768, 64, "residual"), (8300, 256, 32, "store_f32")])
@pytest.mark.parametrize("dtype", DTYPES)
def test_tiles_and_splits(dtype, M, N, K, group, epilogue):
    announce("quant tiles", dtype, M, N, K, group, epilogue)
    inputs = product_inputs(M, N, K, group, True, epilogue, dtype, M + N)
    check_product(*inputs, epilogue, run_product(*inputs, epilogue, N))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,N,K,group,epilogue", [(1, 16500, 64, 32, "store"), (9, 8200, 128, 64, "swiglu"), (16, 2100, 192, 64, "residual"), (4, 4100, 320, 32, "store"),
                                                  (300, 96, 256, 128, "store"), (1025, 40, 96, 32, "residual")])
def test_wide_few_rows_and_many_rows(dtype, M, N, K, group, epilogue):
    announce("quant wide", dtype, M, N, K, group, epilogue)
    inputs = product_inputs(M, N, K, group, True, epilogue, dtype, M + N)
    check_product(*inputs, epilogue, run_product(*inputs, epilogue, N))


@pytest.mark.parametrize("M,N,K,group", [(20, 8200, 4128, 32), (40, 8200, 5152, 32), (20, 8200, 7232, 64), (10, 16500, 4128, 32)])
def test_scales_brought_in_parts(M, N, K, group):
    """More groups than LDS holds the scales of at a time, a last step that is partly filled."""
    announce("quant many groups", M, N, K, group)
    inputs = product_inputs(M, N, K, group, True, "store_f32", torch.bfloat16, M + N)
    check_product(*inputs, "store_f32", run_product(*inputs, "store_f32", N))


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_workspace_of_the_caller_s(dtype):
    inputs = product_inputs(33, 100, 4096, 64, True, "store", dtype, 2)
    x, codes, scales, z, _ = (t.cuda() if t is not None else None for t in inputs)
    need = A.atts_gemm_nt_quant_workspace_bytes(dtype, 33, 100, 4096, A.EPILOGUE_STORE)
    announce("quant workspace", dtype, need)
    out = [torch.empty(33, 100, dtype=dtype, device="cuda") for _ in range(2)]
    A.atts_gemm_nt_quant(x, codes, scales, z, out[0])
    A.atts_gemm_nt_quant(x, codes, scales, z, out[1], workspace=dirty_ws(max(need, 256)))
    assert need > 0 and torch.equal(*out)
    with pytest.raises(A.AttsError) as e:
        A.atts_gemm_nt_quant(x, codes, scales, z, out[1], workspace=dirty_ws(need)[:need - 256])
    assert e.value.code == A.ERR_WORKSPACE


@pytest.mark.parametrize("dtype", DTYPES)
def test_appends_of_many_short_sequences(dtype):
    """More than 64 sequences in one workgroup's rows, most of them without any."""
    announce("append sparse", dtype)
    lens = [1 if s % 40 == 3 else 0 for s in range(2000)]
    append_case(lens, [s % 37 for s in range(2000)], 2, 1, 32, 32, 16, dtype, False, seed=4)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lens,cached,page,softcap,window", [([70, 1], [700, 5], 16, 0.0, 0), ([5], [3000], 64, 20.0, 1000), ([256], [257], 8, 0.0, 100)])
def test_heads_of_256(dtype, lens, cached, page, softcap, window):
    announce("tree heads of 256", dtype, lens, cached, page, softcap, window)
    p, kv, q, parents = tree_inputs(lens, cached, 6, 2, 256, page, dtype, "branches", seed=sum(lens))
    got = run_tree(p, q, parents, cached, lens, softcap=softcap, window=window)
    check_tree(got, q, kv, parents, cached, lens, 6, 256, dtype, softcap=softcap, window=window)


@pytest.mark.parametrize("dtype", DTYPES)
def test_trees_of_many_sequences(dtype):
    rng = np.random.default_rng(5)
    lens, cached = [int(n) for n in rng.integers(0, 9, 200)], [int(c) for c in 2 ** rng.uniform(0, 9, 200)]
    announce("tree 200 sequences", dtype)
    p, kv, q, parents = tree_inputs(lens, cached, 4, 4, 32, 16, dtype, "branches", seed=12)
    check_tree(run_tree(p, q, parents, cached, lens), q, kv, parents, cached, lens, 4, 32, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
def test_scores_of_the_lowest_values(dtype):
    """Finite keys whose scores come out as -inf have no weight, wherever they lie; a row that sees no other key gives zeros."""
    hd, big, n_low = 8, torch.finfo(dtype).max, 1500               # whole tiles and splits of them, then keys that score 0
    g = torch.Generator().manual_seed(1)
    announce("tree lowest scores", dtype)
    for context in (1500, 1501, 2100):
        p = Paged(np.random.default_rng(0), [context + 3], 1, 8, hd, dtype)
        k, v = torch.full((context + 3, 1, hd), -big, dtype=dtype), torch.randn(context + 3, 1, hd, generator=g).to(dtype)
        k[n_low:context], k[context + 1] = 0.0, 0.0
        p.fill_sequence(0, k, v)
        got = host(run_tree(p, torch.full((3, hd), big, dtype=dtype), [[-1, -1, 1]], [context], [3]))
        rest, seen = host(v)[n_low:context, 0].astype(np.float64), host(v)[context + 1, 0].astype(np.float64)
        both = np.concatenate([rest, seen[None]]).mean(axis=0)     # equal weights: sums of up to 601 values in 32 bits; 16 bits: one rounding
        tol = 4 * UNIT[dtype] * np.abs(host(v)).max()
        assert np.abs(got[0] - (rest.mean(axis=0) if len(rest) else 0.0)).max() <= tol and np.abs(got[1:] - both).max() <= tol


def test_a_cache_past_32_bits():
    """Pages behind element 2^31 of the keys and values (2 x 4.4 GB): appended to, read, and nothing else written."""
    n_pages, nkv, page, hd = 70000, 2, 128, 128                    # 2.29e9 elements each
    k = torch.zeros(n_pages, nkv, page, hd, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros(n_pages, nkv, hd, page, dtype=torch.bfloat16, device="cuda")
    cache = A.PagedCache(k, v, i32([[69999, 1], [4463, 69998]]))   # 4463 and 69999 are 65,536 pages apart: 2^31 elements
    g = torch.Generator().manual_seed(3)
    lens, cached, nq = [140, 130], [0, 0], 4
    qkv = torch.randn(270, (nq + 2 * nkv) * hd, generator=g).bfloat16()
    q, table = torch.empty(270, nq * hd, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, hd // 2, 2, device="cuda")
    table[..., 0] = 1.0                                            # no rotation
    announce("cache past 32 bits")
    A.atts_rotary_append(cache, qkv.cuda(), i32([0] * 270), i32(cached), i32(offsets(lens)), table, A.ROTARY_HALF, q)
    y = qkv.reshape(270, nq + 2 * nkv, hd)
    for first, n, pages in ((0, 140, (69999, 1)), (140, 130, (4463, 69998))):
        for at in range(0, n, 128):
            m = min(128, n - at)
            rows = y[first + at:first + at + m]
            assert torch.equal(k[pages[at // 128], :, :m].cpu(), rows[:, nq:nq + nkv].transpose(0, 1))
            assert torch.equal(v[pages[at // 128], :, :, :m].cpu(), rows[:, nq + nkv:].permute(1, 2, 0))
    assert sum(int(torch.count_nonzero(k[at:at + 10000].any(dim=3))) for at in range(0, n_pages, 10000)) == 270 * nkv
    parents, cached = [list(range(-1, 9)), [-1, 0]], [130, 128]    # trees over what was appended
    out = torch.empty(12, nq * hd, dtype=torch.bfloat16, device="cuda")
    q2 = torch.cat([q[130:140], q[268:270]]).contiguous()
    A.atts_attention_tree(cache, q2, i32(parents[0] + parents[1]), i32(cached), i32([0, 10, 12]), 10, 130, out,
                          ws(A.atts_attention_tree_workspace_bytes(cache, nq, 12, 10, 130)))
    kv = [tuple(host(y[f:f + n, nq + s:nq + s + nkv]) for s in (0, nkv)) for f, n in ((0, 140), (140, 130))]
    check_tree(out, q2, kv, parents, cached, [10, 2], nq, hd, torch.bfloat16)


def test_captured_and_replayed():
    """A step in one graph: every replay, on inputs that changed in place, gives what the eager calls give, with eager work in between."""
    dt, nq, nkv, hd, lens, V, d = torch.bfloat16, 4, 2, 64, [5, 3, 1], 3000, 256
    R, rng, g = sum(lens), np.random.default_rng(1), torch.Generator(device="cuda").manual_seed(2)
    r = lambda *shape: torch.randn(*shape, device="cuda", generator=g)
    wide = (nq + 2 * nkv) * hd
    codes, zeros = (torch.randint(0, top, (wide, n), dtype=torch.uint8, device="cuda", generator=g) for top, n in ((256, d // 2), (16, d // 64)))
    scales, x, logits = (r(wide, d // 64).abs() / 70).to(dt), r(40, d).to(dt), r(R, V)
    p = Paged(rng, [1000] * 3, nkv, 16, hd, dt, fill=0.5)
    parents, off, cached, pos = i32([t for n in lens for t in tree(rng, n)]), i32(offsets(lens)), i32([900, 0, 37]), i32(np.arange(R))
    rotary, params, history = r(64, hd // 2, 2), torch.rand(3, 4, device="cuda", generator=g) + 0.5, i32(rng.integers(0, V, 90))
    spaces = [ws(max(256, n)) for n in (A.atts_gemm_nt_quant_workspace_bytes(dt, 40, wide, d, A.EPILOGUE_STORE),
                                        A.atts_attention_tree_workspace_bytes(p.cache, nq, R, 5, 1000), A.atts_logits_adjust_workspace_bytes(R, V))]
    outs = [torch.empty(40, wide, dtype=dt, device="cuda"), torch.empty(R, nq * hd, dtype=dt, device="cuda"), torch.empty(R, nq * hd, dtype=dt, device="cuda"),
            torch.empty_like(logits), i32([0] * R), torch.empty(R, device="cuda")]

    def step():
        A.atts_gemm_nt_quant(x, codes, scales, zeros, outs[0], workspace=spaces[0])
        A.atts_rotary_append(p.cache, outs[0][:R], pos, cached, off, rotary, A.ROTARY_HALF, outs[1])
        A.atts_attention_tree(p.cache, outs[1], parents, cached, off, 5, 1000, outs[2], spaces[1])
        A.atts_logits_adjust(logits, off, params, history, i32_h, split, pos, parents, None, None, None, None, outs[3], outs[4], outs[5], spaces[2], max_rows=5)
    i32_h, split = i32([0, 30, 60, 90]), i32([10, 0, 30])
    announce("step in a graph")
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(4):
        x.copy_(r(40, d))
        logits.copy_(r(R, V))
        cached.copy_(i32([900 - 100 * turn, turn, 37]))
        for t in outs + spaces:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs] + [p.k.clone(), p.v.clone()]
        for t in outs + spaces:
            t.fill_(1)
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, outs + [p.k, p.v])), turn
