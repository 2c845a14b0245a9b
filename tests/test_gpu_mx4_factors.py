"""Products of NVFP4 matrices whose row factors lie far apart, or leave fp32's range when they are multiplied with each other."""
import numpy as np
import pytest
import torch

from tests import mx4_reference as ref

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
# exponents of the tokens' and of the weights' factors
FAR = {"product_is_zero": ([-80, -83], [-75, -71]), "product_is_subnormal": ([-70, -66], [-69, -72]), "product_is_infinite": ([70, 66], [61, 60]),
       "far_apart": ([100, -30, 0], [-126, -118]), "subnormal_factor": ([-140, -149, -130], [20, 3]),
       "all_kinds": ([-120, -75, -20, 0, 30, 90, 120], [-126, -90, -40, 0, 45, 70, 110])}


@pytest.fixture(scope="module")
def m():
    import paper_2406_13868_b200 as mod
    mod.lib()
    return mod


def matrix(m, g, R, K, exponents, zeros, round_factors):
    """random codes and scales of all magnitudes, `zeros`: slice of K that holds nothing in every third row"""
    codes = torch.randint(0, 16, (R, K), generator=g, dtype=torch.uint8)
    codes[::3, zeros] = 0
    scales = torch.randint(1, 127, (R, -(-K // 16)), generator=g, dtype=torch.uint8)
    scales[1::4] = torch.randint(1, 9, scales[1::4].shape, generator=g, dtype=torch.uint8)          # rows of the smallest scales
    e = torch.tensor(exponents, dtype=torch.float64)[torch.arange(R) % len(exponents)]
    f = torch.exp2(e) * (1.0 if round_factors else 1 + torch.rand(R, generator=g, dtype=torch.float64))
    f = f.to(torch.float32)
    q = m.sdq_mx4_import(torch.from_numpy(ref.pack(codes.numpy())).cuda(), scales.cuda(), m.FMT_NVFP4, K=K, factor=f.cuda())
    return q, ref.values(codes.numpy(), scales.numpy(), np.ones(R), True), f.double().numpy()


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("kind", list(FAR))
@pytest.mark.parametrize("M,N,K", [(3, 130, 48), (40, 300, 1040), (700, 520, 48), (1300, 256, 512), (600, 333, 1040)])
def test_factors_are_applied_without_leaving_the_range(m, M, N, K, kind, dtype):
    g = torch.Generator().manual_seed(M + N + K)
    (xq, xv, fx), (wq, wv, fw) = (matrix(m, g, R, K, FAR[kind][i], slice(0, K // 2) if i else slice(K // 2, K), M % 2 == 0) for i, R in enumerate((M, N)))
    bias = None if kind == "all_kinds" else torch.zeros(N, dtype=DT[dtype], device="cuda")
    got = m.sdq_mx4_linear(xq, wq, bias=bias, dtype=DT[dtype])
    assert m.device_status() == 0
    got = got.double().cpu().numpy()
    s, f = xv @ wv.T, fx[:, None] * fw[None, :]
    # products are exact and a sum of K of them in fp32 is within K 2^-23 of the sum of their magnitudes; then at most three roundings, and the
    # output's, which is half of the smallest number where it is subnormal
    eps, least = (2.0 ** -8, 2.0 ** -134) if dtype == "bf16" else (2.0 ** -24, 2.0 ** -150)
    want, err = s * f, K * 2.0 ** -23 * (np.abs(xv) @ np.abs(wv).T) * f
    tol = err + (2.0 ** -22 + eps * 1.01) * (np.abs(want) + err) + 2 * least
    assert not np.isnan(got).any()                         # (a sum of zero stays zero, whatever its factors are)
    top = float(torch.finfo(DT[dtype]).max)
    fits = np.abs(want) + tol < top
    assert fits.any() and (np.abs(got - want)[fits] <= tol[fits]).all()
    gone = np.abs(want) - tol > top
    assert np.isinf(got[gone]).all()
    assert (got[::3, ::3] == 0).all()


@pytest.mark.parametrize("M", [5, 40, 700])
def test_quantized_rows_of_tiny_and_of_huge_numbers(m, M):
    """rows near 2^-68 against rows near 2^-66, whose factors' product is zero in fp32, give outputs above 2^-126; rows with one huge channel each, not the same one, give zero"""
    g = torch.Generator().manual_seed(M)
    K, N = 2048, 256
    x, w = (1 + torch.rand(R, K, generator=g) for R in (M, N))
    xq, wq = m.sdq_mx4_quantize((x * 2.0 ** -68).cuda(), m.FMT_NVFP4), m.sdq_mx4_quantize((w * 2.0 ** -66).cuda(), m.FMT_NVFP4)
    xv, wv = (m.sdq_mx4_dequantize(q, torch.float32).cpu().double().numpy() for q in (xq, wq))
    want = xv @ wv.T
    got = m.sdq_mx4_linear(xq, wq, dtype=torch.float32).double().cpu().numpy()
    assert want.min() > 2.0 ** -126 and (np.abs(got - want) <= (K * 2.0 ** -23 + 2.0 ** -22) * want + 2.0 ** -149).all()
    x, w = torch.zeros(M, K), torch.zeros(N, K)
    x[:, 7], w[:, 9] = 2.0 ** 120, 2.0 ** 100
    y = m.sdq_mx4_linear(m.sdq_mx4_quantize(x.cuda(), m.FMT_NVFP4), m.sdq_mx4_quantize(w.cuda(), m.FMT_NVFP4))
    assert (y == 0).all()
    assert m.device_status() == 0
