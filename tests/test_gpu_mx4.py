"""Plain microscaled 4-bit matrices on the GPU against their definition in 64 bits (tests/mx4_reference.py)."""
import numpy as np
import pytest
import torch

from tests import mx4_reference as ref

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def m():
    import paper_2406_13868_b200 as mod
    mod.lib()
    return mod


def inputs(R, K, dtype, seed, spread=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(R, K, generator=g)
    if spread:
        x *= torch.exp2(torch.randint(-12, 12, (R, 1), generator=g).float())
        x *= torch.exp2(torch.randint(-3, 4, (R, K), generator=g).float())
        x[torch.rand(R, K, generator=g) < 0.05] = 0
    return x.clamp(-6e4, 6e4).to(dtype)


def as64(x):
    return x.detach().cpu().double().numpy()


def check_quantized(m, q, x, nv, ceil_rule):
    """codes, scales, factors and values of a quantized matrix are the definition's, bit for bit"""
    codes, scales, factor = ref.quantize(as64(x), nv, ceil_rule, float(torch.finfo(x.dtype).max))
    e = {k: v.cpu().numpy() for k, v in m.mx4_export(q).items()}
    got = ref.unpack(e["code"], x.shape[1])
    nan = np.repeat(scales == (127 if nv else 255), 16 if nv else 32, 1)[:, :x.shape[1]]
    assert np.array_equal(e["scale"], scales)
    assert np.array_equal(np.where(nan, 0, got), np.where(nan, 0, codes))
    if nv:
        assert np.array_equal(e["factor"], factor.astype(np.float32))
    if x.shape[1] % 2:
        assert not (e["code"][:, -1] >> 4).any()
    want = ref.values(got, scales, factor, nv)
    for dt in DT.values():
        with np.errstate(over="ignore"):
            w = torch.from_numpy(want).to(torch.float32).to(dt)         # (the values have at most seven significant bits: fp32 holds them)
        y = m.sdq_mx4_dequantize(q, dt).cpu()
        assert torch.equal(torch.isnan(y), torch.isnan(w)) and torch.equal(torch.nan_to_num(y.float()), torch.nan_to_num(w.float()))


@pytest.mark.parametrize("nv,ceil_rule", [(False, False), (False, True), (True, False)])
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("R,K", [(1, 1), (1, 4096), (3, 15), (8, 128), (9, 129), (127, 640), (130, 257), (33, 2056), (5, 4109), (2, 16400)])
def test_quantize_is_the_definition(m, nv, ceil_rule, dtype, R, K):
    x = inputs(R, K, DT[dtype], R * 1000 + K)
    q = m.sdq_mx4_quantize(x.cuda(), m.FMT_NVFP4 if nv else m.FMT_MXFP4, m.SCALE_CEIL_NOSAT if ceil_rule else m.SCALE_OCP_FLOOR)
    check_quantized(m, q, x, nv, ceil_rule)
    assert m.device_status() == 0


@pytest.mark.parametrize("nv,ceil_rule", [(False, False), (False, True), (True, False)])
@pytest.mark.parametrize("dtype", list(DT))
def test_ties_extremes_and_zeros(m, nv, ceil_rule, dtype):
    """element quotients on and beside every boundary, block maxima on scale boundaries, the ends of the types' ranges"""
    dt = DT[dtype]
    fi = torch.finfo(dt)
    mids = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0])
    rows = []
    for e in (-14, -3, 0, 5):
        for s in (1.0, 1.125, 1.375, 1.875):
            v = (mids * s * 2.0 ** e).to(dt)
            near = torch.cat([v, torch.nextafter(v, torch.zeros_like(v)), torch.nextafter(v, torch.full_like(v, fi.max))]) if dt == torch.float32 else \
                torch.cat([v, v * (1 - fi.eps), v * (1 + fi.eps)]).to(dt)
            r = torch.zeros(64, dtype=dt)
            r[:near.numel()] = near
            r[40] = 6 * s * 2.0 ** e
            r[50:58] = -v[:8]
            rows.append(r)
    for a in (fi.max, fi.tiny, fi.smallest_normal / 2 if dt == torch.float32 else fi.tiny, 2688.0, 2689.0, 448.0 * 6 / 4, 0.0):
        r = torch.zeros(64, dtype=dt)
        r[0], r[33] = a, -a
        r[1:9] = torch.tensor([a / 7, a / 3, -a / 2, a / 5, 0, -0.0, a / 100, a / 4096]).to(dt)
        rows.append(r)
    for k in range(8, 64):                                              # block maxima at and between E4M3 multiples of 6
        r = torch.zeros(64, dtype=dt)
        r[0], r[16], r[32], r[48] = 2688.0, 6 * k / 16 * 4, 6 * (2 * k + 1) / 32 * 4, 6 * (2 * k + 1) / 32 / 64
        rows.append(r)
    x = torch.stack(rows).to(dt)
    q = m.sdq_mx4_quantize(x.cuda(), m.FMT_NVFP4 if nv else m.FMT_MXFP4, m.SCALE_CEIL_NOSAT if ceil_rule else m.SCALE_OCP_FLOOR)
    check_quantized(m, q, x, nv, ceil_rule)


@pytest.mark.parametrize("nv", [False, True])
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("K", [96, 77])
def test_infinities_saturate_and_nan_marks_its_block(m, nv, dtype, K):
    x = inputs(12, K, DT[dtype], 3, spread=False)
    x[0, 5] = float("inf")
    x[1, 40] = -float("inf")
    x[2, 3] = float("nan")
    x[3, 50], x[3, 60] = float("nan"), float("inf")
    q = m.sdq_mx4_quantize(x.cuda(), m.FMT_NVFP4 if nv else m.FMT_MXFP4)
    check_quantized(m, q, x, nv, False)


@pytest.mark.parametrize("nv", [False, True])
def test_strided_rows_own_buffers_and_untouched_surroundings(m, nv):
    fmt = m.FMT_NVFP4 if nv else m.FMT_MXFP4
    big = inputs(40, 700, torch.bfloat16, 7).cuda()
    for lo, K in ((0, 256), (8, 320), (3, 301)):                          # aligned, aligned with an offset, of no alignment
        x = big[2:35, lo:lo + K]
        check_quantized(m, m.sdq_mx4_quantize(x, fmt), x.cpu(), nv, False)
        n = m.mx4_size(33, K, fmt)
        buf = torch.full((n + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
        q = m.sdq_mx4_quantize(x, fmt, buf=buf)
        assert q.buf is buf and (buf[n:] == 0xA5).all()
        out = torch.full((33, K + 9), 7.0, dtype=torch.bfloat16, device="cuda")
        m.sdq_mx4_dequantize(q, out=out[:, 4:4 + K])
        assert (out[:, :4] == 7).all() and (out[:, 4 + K:] == 7).all()
        assert torch.equal(out[:, 4:4 + K], m.sdq_mx4_dequantize(q))


@pytest.mark.parametrize("nv", [False, True])
@pytest.mark.parametrize("R,K", [(1, 1), (5, 33), (130, 300), (257, 512)])
def test_import_and_export_are_each_other_s_reverse(m, nv, R, K):
    g = torch.Generator().manual_seed(R + K)
    codes = torch.randint(0, 256, (R, (K + 1) // 2), generator=g, dtype=torch.uint8)
    if K % 2:
        codes[:, -1] &= 15
    n = 16 if nv else 32
    scales = torch.randint(0, 127 if nv else 255, (R, -(-K // n)), generator=g, dtype=torch.uint8)
    factor = torch.rand(R, generator=g) + 0.5 if nv else None
    q = m.sdq_mx4_import(codes.cuda(), scales.cuda(), m.FMT_NVFP4 if nv else m.FMT_MXFP4, K=K, factor=None if factor is None else factor.cuda())
    e = m.mx4_export(q)
    assert torch.equal(e["code"].cpu(), codes) and torch.equal(e["scale"].cpu(), scales)
    if nv:
        assert torch.equal(e["factor"].cpu(), factor)
        assert (m.mx4_export(m.sdq_mx4_import(codes.cuda(), scales.cuda(), m.FMT_NVFP4, K=K))["factor"] == 1).all()


@pytest.mark.parametrize("E,R,K", [(1, 1, 1), (3, 130, 200), (2, 128, 128), (4, 5, 4101)])
def test_experts_hold_what_their_matrices_hold(m, E, R, K):
    w = inputs(E * R, K, torch.bfloat16, E + K).view(E, R, K)
    q = m.sdq_mx4_experts(w.cuda(), m.SCALE_CEIL_NOSAT)
    e = m.mx4_export(q)
    for i in range(E):
        one = m.mx4_export(m.sdq_mx4_quantize(w[i].cuda(), m.FMT_MXFP4, m.SCALE_CEIL_NOSAT))
        assert torch.equal(e["code"][i], one["code"]) and torch.equal(e["scale"][i], one["scale"])
    again = m.sdq_mx4_experts_import(e["code"], e["scale"], K=K)
    assert torch.equal(again.buf, q.buf)                                   # padding included: all of the buffer is defined
    assert torch.equal(m.sdq_mx4_dequantize(q)[E - 1], m.sdq_mx4_dequantize(m.sdq_mx4_quantize(w[E - 1].cuda(), m.FMT_MXFP4, m.SCALE_CEIL_NOSAT)))


# ---- product ---------------------------------------------------------------------------------------------------------------
def linear_case(m, M, N, K, nv, dtype, bias, seed=0, out=None):
    fmt = m.FMT_NVFP4 if nv else m.FMT_MXFP4
    x, w = inputs(M, K, torch.bfloat16, seed + 1), inputs(N, K, torch.bfloat16, seed + 2)
    b = inputs(1, N, DT[dtype], seed + 3, spread=False)[0] if bias else None
    xq, wq = m.sdq_mx4_quantize(x.cuda(), fmt), m.sdq_mx4_quantize(w.cuda(), fmt)
    y = m.sdq_mx4_linear(xq, wq, bias=None if b is None else b.cuda(), dtype=DT[dtype], out=out)
    assert m.device_status() == 0
    xv, wv = as64(m.sdq_mx4_dequantize(xq, torch.float32)), as64(m.sdq_mx4_dequantize(wq, torch.float32))
    want = xv @ wv.T + (0 if b is None else as64(b))
    # products are exact; a sum of K of them in fp32, whatever its order and also where terms are cut rather than rounded, is within
    # K 2^-23 of the sum of the magnitudes; factors, bias and output round once each
    scale = np.abs(xv) @ np.abs(wv).T
    eps = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11, "fp32": 2.0 ** -24}[dtype]
    tol = K * 2.0 ** -23 * scale + 2.0 ** -22 * (np.abs(want) + scale) + eps * np.abs(want) * 1.01 + (2.0 ** -24 if dtype == "fp16" else 1e-40)
    got = as64(y)
    top = float(torch.finfo(DT[dtype]).max)
    fits = np.abs(want) + tol < top
    assert np.isfinite(got[fits]).all()
    assert (np.abs(got - want)[fits] <= tol[fits]).all(), np.max((np.abs(got - want) / tol)[fits])
    return y, xq, wq


@pytest.mark.parametrize("nv", [False, True])
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 128, 256), (1, 256, 4096), (3, 130, 300), (16, 384, 1024), (17, 200, 777), (64, 129, 2048), (100, 1000, 513), (128, 128, 8192),
                                   (129, 300, 260), (333, 520, 1030), (512, 256, 512)])
def test_linear_few_tokens(m, nv, M, N, K):
    linear_case(m, M, N, K, nv, "fp32", False)


@pytest.mark.parametrize("nv", [False, True])
@pytest.mark.parametrize("M,N,K", [(513, 128, 256), (513, 1, 1), (520, 300, 700), (768, 512, 4096), (1025, 1000, 513), (2048, 2304, 300), (4100, 520, 260)])
def test_linear_many_tokens(m, nv, M, N, K):
    linear_case(m, M, N, K, nv, "fp32", False)


@pytest.mark.parametrize("nv", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("M,N,K", [(5, 300, 500), (200, 256, 512), (600, 320, 640), (700, 333, 257)])
def test_linear_types_and_bias(m, nv, dtype, bias, M, N, K):
    linear_case(m, M, N, K, nv, dtype, bias)


@pytest.mark.parametrize("M", [4, 600])
@pytest.mark.parametrize("pad", [0, 1, 16])
def test_linear_into_part_of_a_larger_output(m, M, pad):
    big = torch.full((M + 2, 320 + 2 * pad), 7.0, dtype=torch.bfloat16, device="cuda")
    view = big[1:M + 1, pad:pad + 320]
    y, xq, wq = linear_case(m, M, 320, 512, False, "bf16", False, out=view)
    assert y is view and torch.equal(view, m.sdq_mx4_linear(xq, wq))
    assert (big[0] == 7).all() and (big[-1] == 7).all() and (big[:, :pad] == 7).all() and (pad == 0 or (big[:, pad + 320:] == 7).all())


@pytest.mark.parametrize("M", [2, 700])
def test_linear_nan_reaches_its_row_only(m, M):
    x = inputs(M, 600, torch.bfloat16, 1, spread=False)
    x[1, 599] = float("nan")
    y = m.sdq_mx4_linear(m.sdq_mx4_quantize(x.cuda()), m.sdq_mx4_quantize(inputs(300, 600, torch.bfloat16, 2).cuda()))
    assert torch.isnan(y[1]).all() and torch.isfinite(y[torch.arange(M) != 1]).all()


@pytest.mark.parametrize("M", [1, 40, 300, 900])
def test_linear_gives_the_same_bits_again_and_for_each_row_alone(m, M):
    y, xq, wq = linear_case(m, M, 640, 2048, True, "fp32", False)
    for _ in range(3):
        assert torch.equal(y, m.sdq_mx4_linear(xq, wq, dtype=torch.float32))


def test_linear_factors_of_a_checkpoint(m):
    """any fp32 factor, one for all rows as a per-tensor scale is"""
    g = torch.Generator().manual_seed(5)
    w = m.mx4_export(m.sdq_mx4_quantize(inputs(200, 512, torch.bfloat16, 2).cuda(), m.FMT_NVFP4))
    f = torch.full((200,), 0.0137, device="cuda")
    wq = m.sdq_mx4_import(w["code"], w["scale"], m.FMT_NVFP4, factor=f)
    x = torch.randn(7, 512, generator=g).cuda()
    xq = m.sdq_mx4_quantize(x, m.FMT_NVFP4)
    want = as64(m.sdq_mx4_dequantize(xq, torch.float32)) @ ref.values(ref.unpack(w["code"].cpu().numpy(), 512), w["scale"].cpu().numpy(), as64(f), True).T
    y = as64(m.sdq_mx4_linear(xq, wq, dtype=torch.float32))
    assert np.abs(y - want).max() <= 1e-5 * np.abs(want).max()


def test_streams_captures_and_concurrent_calls(m):
    """a captured quantize + product replays on new inputs; calls on two streams at once do not share anything"""
    x = inputs(24, 1024, torch.bfloat16, 1).cuda()
    wq = m.sdq_mx4_quantize(inputs(512, 1024, torch.bfloat16, 2).cuda())
    want = m.sdq_mx4_linear(m.sdq_mx4_quantize(x), wq)
    static, out = x.clone(), torch.empty_like(want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        m.sdq_mx4_linear(m.sdq_mx4_quantize(static), wq, out=out)
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        m.sdq_mx4_linear(m.sdq_mx4_quantize(static), wq, out=out)
    static.copy_(x.flip(0))
    g.replay()
    assert torch.equal(out, want.flip(0))
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    torch.cuda.synchronize()
    for i in range(20):
        with torch.cuda.stream(streams[i % 2]):
            outs.append(m.sdq_mx4_linear(m.sdq_mx4_quantize(x if i % 2 else static), wq))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want if i % 2 else want.flip(0)) for i, o in enumerate(outs))


def test_weights_quantized_right_in_front_of_the_product(m):
    """the launch in front of a product may be the one that writes its weights"""
    x, ws = inputs(8, 4096, torch.bfloat16, 1).cuda(), [inputs(4096, 4096, torch.bfloat16, 2 + i).cuda() for i in range(2)]
    buf = torch.empty(m.mx4_size(4096, 4096), dtype=torch.uint8, device="cuda")
    xq = m.sdq_mx4_quantize(x)
    want = [m.sdq_mx4_linear(xq, m.sdq_mx4_quantize(w)) for w in ws]
    for _ in range(10):
        for i in (0, 1):
            assert torch.equal(m.sdq_mx4_linear(xq, m.sdq_mx4_quantize(ws[i], buf=buf)), want[i])


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("R,K,pad", [(515, 8200, 0), (400, 12000, 8), (261, 16400, 0), (200, 24576, 16)])
def test_many_long_rows_are_quantized_like_few(m, dtype, R, K, pad):
    """rows streamed through shared memory (four and two at a time, ragged ends) against the same rows in calls of their own"""
    x = inputs(R, K + pad, DT[dtype], R).cuda()[:, :K]
    x[3, 17], x[R - 1, K - 1], x[7, 100] = float("nan"), float("inf"), -float("inf")
    a = m.mx4_export(m.sdq_mx4_quantize(x, m.FMT_NVFP4))
    for lo, hi in ((0, 9), (R - 11, R)):
        b = m.mx4_export(m.sdq_mx4_quantize(x[lo:hi], m.FMT_NVFP4))
        nan = torch.repeat_interleave(b["scale"] == 127, 8, 1)[:, :b["code"].shape[1]]
        assert torch.equal(a["scale"][lo:hi], b["scale"]) and torch.equal(a["factor"][lo:hi], b["factor"])
        assert torch.equal(torch.where(nan, 0, a["code"][lo:hi]), torch.where(nan, 0, b["code"]))
    check = x[:40].cpu()
    check_quantized(m, m.sdq_mx4_quantize(x[:40], m.FMT_NVFP4), check, True, False)
    assert m.device_status() == 0


def test_beside_the_decomposed_layers(m):
    """both kinds of products one behind the other in a stream, and in two streams at once, give what each gives alone"""
    K, N = 1024, 1280
    g = torch.Generator().manual_seed(21)
    W = (torch.randn(N, K, generator=g) * 0.02).bfloat16().cuda()
    cfg = m.Config(out_n=1, in_gran=m.GRAN_PAIR, in_block=64, scale_rule=m.SCALE_OCP_FLOOR)
    P, Q = m.sdq_decompose(W, cfg), m.sdq_mx4_quantize(W, m.FMT_NVFP4)
    for M in (2, 40, 128, 300):
        X = torch.randn(M, K, generator=g).bfloat16().cuda()

        def old():
            return m.sdq_linear(m.sdq_quantize_act(X, cfg), P)

        def new():
            return m.sdq_mx4_linear(m.sdq_mx4_quantize(X, m.FMT_NVFP4), Q)

        torch.cuda.synchronize()
        a = old()
        torch.cuda.synchronize()
        b = new()
        torch.cuda.synchronize()
        xa, xb = m.sdq_quantize_act(X, cfg), m.sdq_mx4_quantize(X, m.FMT_NVFP4)
        turns = [f() for _ in range(10) for f in (old, new, lambda: m.sdq_linear(xa, P), lambda: m.sdq_mx4_linear(xb, Q))]
        streams = [torch.cuda.Stream() for _ in range(2)]
        torch.cuda.synchronize()
        for i in range(20):
            for s, f in zip(streams, (old, new)):
                with torch.cuda.stream(s):
                    turns.append(f())
        torch.cuda.synchronize()
        assert all(torch.equal(y, b if i % 2 else a) for i, y in enumerate(turns))
    assert m.device_status() == 0
