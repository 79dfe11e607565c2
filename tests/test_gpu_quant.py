"""Products with 4-bit weights against the 64-bit oracle: every epilogue and type, group sizes, one row to more than a tile, sizes that fill no tile."""
import numpy as np
import pytest
import torch

import paper_2509_15148_amd as A
from oracle import step_oracle as S
from step_util import DTYPES, UNIT, host
from util import announce

pytestmark = pytest.mark.gpu
EPILOGUES = {"store": A.EPILOGUE_STORE, "store_f32": A.EPILOGUE_STORE_F32, "residual": A.EPILOGUE_RESIDUAL, "swiglu": A.EPILOGUE_SWIGLU}


def _inputs(M, N, K, group, zeros, epilogue, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    rows = 2 * N if epilogue == "swiglu" else N
    x = torch.randn(M, K, generator=g).to(dtype)
    codes = torch.randint(0, 256, (rows, K // 2), generator=g, dtype=torch.uint8)
    scales = ((0.5 + torch.rand(rows, K // group, generator=g)) / (4.6 * K ** 0.5)).to(dtype)
    z = torch.randint(0, 16, (rows, K // group), generator=g, dtype=torch.uint8) if zeros else None
    residual = torch.randn(M, N, generator=g) if epilogue == "residual" else None
    return x, codes, scales, z, residual


def _check(x, codes, scales, z, residual, epilogue, got):
    n = lambda t: None if t is None else host(t)
    ref = S.quant_product(n(x), codes.numpy(), n(scales), None if z is None else z.numpy(), epilogue, n(residual))
    # Sums of up to K terms in 32 bits, the codes shifted by up to 16 while they are summed: a term is at most 31 scale |x|; the roundings of a
    # group's 128 additions and of the additions of the groups come to about sqrt(128 + K / 32) <= 16 units of 2^-24 of the sum of the terms' sizes
    size = np.abs(n(x)).astype(np.float64) @ np.repeat(n(scales).astype(np.float64) * 31.0, x.shape[1] // scales.shape[1], axis=1).T
    tol = 16.0 * 2.0 ** -24 * size
    if epilogue == "swiglu":
        y = n(x).astype(np.float64) @ S.dequantize(codes.numpy(), n(scales), None if z is None else z.numpy()).T
        gate, up = np.split(y, 2, axis=1)
        tg, tu = np.split(tol, 2, axis=1)
        silu = gate / (1.0 + np.exp(-gate))
        tol = 1.1 * tg * (np.abs(up) + tu) + tu * np.abs(silu) + 2.0 ** -20 * np.abs(ref)       # |silu'| < 1.1; exp and the quotient in 32 bits
    store = 2.0 ** -24 if epilogue in ("residual", "store_f32") else UNIT[x.dtype]
    err = np.abs(host(got).astype(np.float64) - ref)
    assert (err <= tol * (1 + store) + store * np.abs(ref) * 1.01 + 1e-30).all(), float((err / (tol + store * np.abs(ref) + 1e-30)).max())


def _run(x, codes, scales, z, residual, epilogue, N):
    dt = torch.float32 if epilogue in ("residual", "store_f32") else x.dtype
    out = torch.full((x.shape[0], N), float("nan"), dtype=dt, device="cuda")
    d = lambda t: None if t is None else t.cuda()
    A.atts_gemm_nt_quant(d(x), d(codes), d(scales), d(z), out, EPILOGUES[epilogue], d(residual))
    return out


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("epilogue", list(EPILOGUES))
@pytest.mark.parametrize("M,N,K,group,zeros", [(1, 1, 32, 32, False), (1, 70, 384, 128, True), (3, 16, 64, 64, False), (5, 129, 640, 128, False),
                                               (16, 48, 256, 32, True), (17, 100, 1152, 64, True), (33, 257, 448, 64, True), (64, 64, 512, 128, True),
                                               (65, 33, 96, 32, False), (130, 130, 1024, 128, True)])
def test_products(dtype, epilogue, M, N, K, group, zeros):
    announce("quant", dtype, epilogue, M, N, K, group, zeros)
    inputs = _inputs(M, N, K, group, zeros, epilogue, dtype, M + N + K)
    _check(*inputs, epilogue, _run(*inputs, epilogue, N))


@pytest.mark.parametrize("M,N,K,group", [(1, 4608, 3584, 128), (16, 1024, 8192, 128), (61, 3584, 2368, 64), (2, 512, 18944, 32), (8, 16400, 256, 128)])
def test_wide_and_deep(M, N, K, group):
    announce("quant wide", M, N, K, group)
    inputs = _inputs(M, N, K, group, True, "store", torch.bfloat16, K)
    _check(*inputs, "store", _run(*inputs, "store", N))


@pytest.mark.parametrize("dtype", DTYPES)
def test_every_code_zero_and_place(dtype):
    """One activation at a time: every k alone reaches the output with its own code, scale and zero, zeros up to 255 among them."""
    N, K, group = 40, 256, 32
    g = torch.Generator().manual_seed(5)
    x = torch.eye(K).to(dtype)
    codes = torch.randint(0, 256, (N, K // 2), generator=g, dtype=torch.uint8)
    scales = torch.rand(N, K // group, generator=g).to(dtype)
    z = torch.randint(0, 256, (N, K // group), generator=g, dtype=torch.uint8)
    announce("quant unit rows", dtype)
    got = host(_run(x, codes, scales, z, None, "store_f32", N))
    want = S.dequantize(codes.numpy(), host(scales), z.numpy()).T
    # one term, two roundings, the shift by up to 16 and a zero up to 255 ahead of them
    assert np.abs(got - want).max() <= 2 * 2.0 ** -24 * (15 + 16 + 255)


def test_strided_rows_and_a_residual_in_place():
    x, codes, scales, z, residual = _inputs(9, 50, 256, 64, True, "residual", torch.bfloat16, 3)
    wide = torch.full((9, 256 + 24), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, :256] = x.cuda()
    out = residual.cuda()
    announce("quant strided, in place")
    A.atts_gemm_nt_quant(wide[:, :256], codes.cuda(), scales.cuda(), z.cuda(), out, A.EPILOGUE_RESIDUAL, out)
    _check(x, codes, scales, z, residual, "residual", out)


@pytest.mark.parametrize("M", [1, 40])
def test_rows_do_not_meet(M):
    """A NaN in one row of X, or in one scale, stays in its row or column."""
    x, codes, scales, z, _ = _inputs(M, 70, 384, 128, True, "store", torch.bfloat16, 4)
    x[M // 2, 100], scales[33, 1] = float("nan"), float("inf")
    announce("quant NaN", M)
    bad = torch.isnan(_run(x, codes, scales, z, None, "store", 70).float()).cpu() | torch.isinf(_run(x, codes, scales, z, None, "store", 70).float()).cpu()
    want = torch.zeros(M, 70, dtype=torch.bool)
    want[M // 2], want[:, 33] = True, True
    assert torch.equal(bad, want)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("symmetric", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_quantizer(dtype, symmetric, group):
    N, K = 37, 384
    w = torch.randn(N, K, generator=torch.Generator().manual_seed(group)).to(dtype)
    w[3, :group] = 0.0
    w[4, :group] = w[4, :group].abs()
    codes = torch.full((N, K // 2), 255, dtype=torch.uint8, device="cuda")
    scales = torch.full((N, K // group), float("nan"), dtype=dtype, device="cuda")
    zeros = None if symmetric else torch.full((N, K // group), 255, dtype=torch.uint8, device="cuda")
    announce("quantize", dtype, symmetric, group)
    A.atts_quantize_rows(w.cuda(), codes, scales, zeros)
    want, scale, zero = S.quantize(host(w), group, symmetric, lambda s: host(torch.from_numpy(s).to(dtype)))
    got = codes.cpu().numpy()
    assert np.array_equal(host(scales), scale)
    assert np.array_equal(got & 15, want[:, 0::2]) and np.array_equal(got >> 4, want[:, 1::2])
    assert symmetric or np.array_equal(zeros.cpu().numpy(), zero)
    back = S.dequantize(got, scale, None if symmetric else zero)
    # half a step; the scale's own rounding moves the outermost codes (up to 15 steps) by as much again
    assert (np.abs(back - host(w)) <= np.repeat(scale, group, axis=1) * (0.5 + 16 * UNIT[dtype]) + 1e-12).all()


def test_refusals():
    x, codes, scales, z, residual = _inputs(4, 32, 128, 32, True, "residual", torch.bfloat16, 1)
    x, codes, scales, z, residual = (t.cuda() for t in (x, codes, scales, z, residual))
    out = torch.empty(4, 32, dtype=torch.bfloat16, device="cuda")

    def refused(code, *a, **k):
        with pytest.raises(A.AttsError) as e:
            A.atts_gemm_nt_quant(*a, **k)
        assert e.value.code == code
    refused(A.ERR_INVALID_ARG, x, codes, scales, z, out, A.EPILOGUE_RESIDUAL, None)
    refused(A.ERR_INVALID_ARG, x, codes, scales, z, out, 7)
    refused(A.ERR_INVALID_ARG, x, codes, scales.float(), z, out)
    refused(A.ERR_INVALID_ARG, x.half(), codes, scales, z, out)
    refused(A.ERR_INVALID_ARG, x, codes[:, :32], scales, z, out)
    refused(A.ERR_INVALID_ARG, x, codes, scales, z[:, :2], out)
    refused(A.ERR_INVALID_ARG, x, codes, scales, z, out.float())
    refused(A.ERR_INVALID_ARG, x.t().contiguous().t(), codes, scales, z, out)
    refused(A.ERR_SHAPE, x, codes, scales[:, :1].repeat(1, 8), z[:, :1].repeat(1, 8), out)                   # groups of 16
    wide = torch.zeros(4, 136, dtype=torch.bfloat16, device="cuda")
    refused(A.ERR_INVALID_ARG, wide[:, 1:129], codes, scales, z, out)                                        # x not aligned
    refused(A.ERR_INVALID_ARG, torch.zeros(4, 130, dtype=torch.bfloat16, device="cuda")[:, :128], codes, scales, z, out)
    refused(A.ERR_INVALID_ARG, x.cpu(), codes, scales, z, out)
    A.atts_gemm_nt_quant(x[:0], codes, scales, z, out[:0])                                                   # no rows: nothing to do
