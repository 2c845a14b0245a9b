"""Products of microscaled 4-bit matrices: rows alone and among others, blocks that are not finite, MXFP4 scales from end to end of their range."""
import numpy as np
import pytest
import torch

from tests import mx4_reference as ref
from tests.test_gpu_mx4 import as64, inputs

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def m():
    import paper_2406_13868_b200 as mod
    mod.lib()
    return mod


@pytest.mark.parametrize("nv", [False, True])
@pytest.mark.parametrize("M,N,K", [(40, 640, 2048), (300, 200, 777), (900, 640, 1024)])
def test_a_row_alone_gives_what_it_gives_among_others(m, nv, M, N, K):
    """other rows may change how K is split, and so the order of a sum, and nothing else"""
    fmt = m.FMT_NVFP4 if nv else m.FMT_MXFP4
    x, w = inputs(M, K, torch.bfloat16, M).cuda(), inputs(N, K, torch.bfloat16, N).cuda()
    wq = m.sdq_mx4_quantize(w, fmt)
    xq = m.sdq_mx4_quantize(x, fmt)
    y = m.sdq_mx4_linear(xq, wq, dtype=torch.float32)
    xv, wv = as64(m.sdq_mx4_dequantize(xq, torch.float32)), as64(m.sdq_mx4_dequantize(wq, torch.float32))
    for r in (0, 1, 31, M // 2, M - 1):
        one = m.sdq_mx4_linear(m.sdq_mx4_quantize(x[r:r + 1], fmt), wq, dtype=torch.float32)
        # twice the bound of a sum of K exact products in fp32, and of the roundings behind it
        assert (np.abs(as64(one[0]) - as64(y[r])) <= (K * 2.0 ** -22 + 2.0 ** -21) * (np.abs(xv[r]) @ np.abs(wv).T) + 1e-40).all()
    for c in (0, 127, N - 1):
        one = m.sdq_mx4_linear(xq, m.sdq_mx4_quantize(w[c:c + 1], fmt), dtype=torch.float32)
        assert (np.abs(as64(one[:, 0]) - as64(y[:, c])) <= (K * 2.0 ** -22 + 2.0 ** -21) * (np.abs(xv) @ np.abs(wv[c])) + 1e-40).all()


@pytest.mark.parametrize("nv", [False, True])
@pytest.mark.parametrize("M,N,K", [(2, 300, 600), (70, 300, 600), (700, 300, 600), (1300, 512, 512)])
def test_a_nan_reaches_its_row_and_its_column_only(m, nv, M, N, K):
    fmt = m.FMT_NVFP4 if nv else m.FMT_MXFP4
    x, w = inputs(M, K, torch.bfloat16, 1, spread=False), inputs(N, K, torch.bfloat16, 2, spread=False)
    clean = m.sdq_mx4_linear(m.sdq_mx4_quantize(x.cuda(), fmt), m.sdq_mx4_quantize(w.cuda(), fmt), dtype=torch.float32)
    assert torch.isfinite(clean).all()
    x[1, K - 1], w[N - 1, 3], w[130, 40] = float("nan"), float("nan"), float("nan")
    y = m.sdq_mx4_linear(m.sdq_mx4_quantize(x.cuda(), fmt), m.sdq_mx4_quantize(w.cuda(), fmt), dtype=torch.float32)
    assert torch.isnan(y[1]).all() and torch.isnan(y[:, N - 1]).all() and torch.isnan(y[:, 130]).all()
    rows, cols = torch.ones(M, dtype=torch.bool), torch.ones(N, dtype=torch.bool)
    rows[1], cols[N - 1], cols[130] = False, False, False
    assert torch.equal(y.cpu()[rows][:, cols], clean.cpu()[rows][:, cols])
    # a block of zeros and a NaN is one, whatever it meets
    z = torch.zeros(M, K)
    z[0, 5] = float("nan")
    y = m.sdq_mx4_linear(m.sdq_mx4_quantize(z.cuda(), fmt), m.sdq_mx4_quantize(torch.zeros(N, K, device="cuda"), fmt))
    assert torch.isnan(y[0]).all() and (y[1:] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("M,N,K", [(5, 130, 96), (40, 256, 1024), (700, 300, 96), (1300, 256, 512)])
@pytest.mark.parametrize("lo,hi", [((0, 20), (230, 250)), ((100, 160), (100, 160)), ((0, 254), (0, 254)), ((240, 254), (2, 20))])
def test_mxfp4_scales_of_all_sizes(m, lo, hi, M, N, K, dtype):
    """one side's blocks near 2^-127, the other's near 2^127, and all of it mixed: products are formed of both scales at once"""
    g = torch.Generator().manual_seed(M + N + K)
    mats = []
    for R, (a, b) in ((M, lo), (N, hi)):
        codes = torch.randint(0, 16, (R, K), generator=g, dtype=torch.uint8)
        scales = torch.randint(a, b + 1, (R, 1), generator=g) + torch.randint(-3, 4, (R, -(-K // 32)), generator=g)
        scales = scales.clamp(0, 254).to(torch.uint8)
        mats.append((m.sdq_mx4_import(torch.from_numpy(ref.pack(codes.numpy())).cuda(), scales.cuda(), K=K), ref.values(codes.numpy(), scales.numpy(), None, False)))
    (xq, xv), (wq, wv) = mats
    y = as64(m.sdq_mx4_linear(xq, wq, dtype=DT[dtype]))
    assert m.device_status() == 0
    want, scale = xv @ wv.T, np.abs(xv) @ np.abs(wv).T
    top = float(torch.finfo(DT[dtype]).max)
    eps, least = (2.0 ** -8, 2.0 ** -134) if dtype == "bf16" else (2.0 ** -24, 2.0 ** -150)
    # products below fp32's smallest number count as one of its steps each
    tol = K * 2.0 ** -23 * scale + (2.0 ** -22 + eps * 1.01) * (np.abs(want) + scale * K * 2.0 ** -23) + K * 2.0 ** -126 + 2 * least
    fits = scale * (1 + K * 2.0 ** -23) + tol < top             # (no partial sum leaves the range)
    assert (np.abs(y - want)[fits] <= tol[fits]).all()
    assert not np.isfinite(y[np.abs(want) - tol > 2 * top]).any()


@pytest.mark.parametrize("nv", [False, True])
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("R,K", [(3, 77), (3, 1), (700, 8201), (5, 4109), (2, 16401)])
def test_padding_is_zero_in_a_nan_s_block_too(m, nv, dtype, R, K):
    """the last byte of an odd row holds one code, whatever its block's scale is"""
    fmt = m.FMT_NVFP4 if nv else m.FMT_MXFP4
    x = inputs(R, K, DT[dtype], K, spread=False)
    x[0, K - 1], x[R - 1, K - 1] = float("nan"), float("nan")
    q = m.sdq_mx4_quantize(x.cuda(), fmt)
    e = m.mx4_export(q)
    assert (e["scale"][0, -1] == (127 if nv else 255)).all() and not (e["code"][:, -1] >> 4).any()
    # and so a matrix that is exported and imported is the same one
    again = m.mx4_export(m.sdq_mx4_import(e["code"], e["scale"], fmt, K=K, factor=e.get("factor")))
    assert torch.equal(again["code"], e["code"]) and torch.equal(again["scale"], e["scale"])
