"""Router and expert layer on the GPU against their definition in 64 bits."""
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


# ---- router ----------------------------------------------------------------------------------------------------------------
def route_reference(x, w, k, bias, sigmoid, renorm, scale=1.0):
    logits = x.double().cpu() @ w.double().cpu().T
    score = torch.sigmoid(logits) if sigmoid else torch.softmax(logits, 1)
    choice = score if bias is None else score + bias.double().cpu()
    order = torch.sort(choice, dim=1, descending=True, stable=True)
    ids = order[1][:, :k]
    p = score.gather(1, ids)
    top = order[0]
    gap = (top[:, :-1] - top[:, 1:]).abs()[:, :k].min().item() if top.shape[1] > 1 else 1.0    # (between neighbours of the chosen)
    return ids.int(), (p / p.sum(1, keepdim=True) if renorm else p) * scale, gap


@pytest.mark.parametrize("sigmoid,bias,renorm", [(False, False, True), (False, True, False), (True, False, False), (True, True, True)])
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("T,H,E,k", [(1, 1, 1, 1), (1, 4096, 64, 6), (2, 100, 7, 7), (9, 257, 33, 5), (64, 1024, 256, 8), (5, 64, 1024, 32), (131, 72, 12, 2)])
def test_route(m, sigmoid, bias, renorm, dtype, T, H, E, k):
    g = torch.Generator().manual_seed(T * 7 + H + E)
    x = torch.randn(T, H, generator=g).to(DT[dtype])
    w = (torch.randn(E, H, generator=g) / H ** 0.5).to(DT[dtype])
    b = 0.1 * torch.randn(E, generator=g) if bias else None
    ids, weights, gap = route_reference(x, w, k, b, sigmoid, renorm, 2.5)
    got, gw = m.sdq_moe_route(x.cuda(), w.cuda(), k, bias=None if b is None else b.cuda(), scoring=m.ROUTE_SIGMOID if sigmoid else m.ROUTE_SOFTMAX,
                              renorm=renorm, scale=2.5)
    assert got.dtype == torch.int32 and gw.dtype == torch.float32
    # fp32: eight products at a time, 16-bit operands: 32 on the tensor core, which may cut what it adds: a logit is off by less than so many
    # times 2^-24 or 2^-23 of the sum of its products' magnitudes, a score by as much
    mag = (x.double().abs() @ w.double().abs().T).max().item()
    err = 2 * (8 * 2.0 ** -24 if dtype == "fp32" else 32 * 2.0 ** -23) * mag
    if gap > err:
        assert torch.equal(got.cpu(), ids)
    else:                                             # two experts nearer to each other than that: k different ones, all the same
        assert all(len(set(r)) == k for r in got.tolist())
    if torch.equal(got.cpu(), ids):
        assert ((gw.cpu().double() - weights).abs() <= (4 * err + 2.0 ** -22) * weights.abs() + 1e-38).all()


def test_route_ties_take_the_lowest_index(m):
    x = torch.ones(3, 16, dtype=torch.bfloat16).cuda()
    x[2] = 0
    w = torch.zeros(40, 16, dtype=torch.bfloat16)
    w[[7, 11, 35, 39]] = 1
    w[[3, 20]] = 0.5
    ids, weights = m.sdq_moe_route(x, w.cuda(), 8)
    assert ids.tolist() == [[7, 11, 35, 39, 3, 20, 0, 1]] * 2 + [list(range(8))]
    assert torch.allclose(weights.sum(1), torch.ones(3, device="cuda")) and (weights[2] == 0.125).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,E,k", [(9, 2, 2), (3, 31, 31), (8, 33, 32), (17, 127, 9), (5, 128, 32), (5, 129, 32), (2, 1000, 32)])
def test_route_order_of_many_ties(m, dtype, T, E, k):
    """logits that are exact small integers: of equal ones the lowest index, up to the number of experts where places are counted and beyond"""
    g = torch.Generator().manual_seed(T + E)
    x, w = (torch.randint(-1, 2, s, generator=g).to(DT[dtype]) for s in ((T, 20), (E, 20)))
    ids, weights = m.sdq_moe_route(x.cuda(), w.cuda(), k, renorm=False)
    logits = x.double() @ w.double().T
    want = torch.sort(logits, dim=1, descending=True, stable=True)[1][:, :k]
    assert torch.equal(ids.cpu().long(), want)
    score = torch.softmax(logits, 1).gather(1, want)
    assert ((weights.cpu().double() - score).abs() <= 2.0 ** -23 * score).all()      # (64-bit scores, rounded once)


@pytest.mark.parametrize("H", [64, 65])
def test_route_strides_and_non_finite_tokens(m, H):
    g = torch.Generator().manual_seed(1)
    x, w = torch.randn(20, 160, generator=g).bfloat16().cuda(), torch.randn(30, 200, generator=g).bfloat16().cuda()
    a = m.sdq_moe_route(x[3:15, 16:16 + H], w[2:25, 8:8 + H], 4)
    b = m.sdq_moe_route(x[3:15, 16:16 + H].contiguous(), w[2:25, 8:8 + H].contiguous(), 4)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    x[4, 20], x[5, 20] = float("nan"), float("inf")
    ids, weights = m.sdq_moe_route(x[3:15, 16:16 + H], w[2:25, 8:8 + H], 4)
    assert torch.isnan(weights[1]).all() and ((ids >= 0) & (ids < 23)).all()
    keep = torch.tensor([0] + list(range(3, 12))).cuda()
    assert torch.equal(ids[keep], a[0][keep]) and torch.equal(weights[keep], a[1][keep])


# ---- expert layer -----------------------------------------------------------------------------------------------------------
def experts(m, E, R, K, seed, size=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = torch.randn(E, R, K, generator=g, device="cuda")
    w = w * (1 + 0.3 * w * w) * ((0.5 / K ** 0.5) if size is None else size)
    q = m.sdq_mx4_experts(w)
    return q, m.sdq_mx4_dequantize(q, torch.float32).double()


def check_moe(m, T, H, I, E, k, dtype, seed=0, ids=None, x=None, out=None, workspace=None):
    g = torch.Generator().manual_seed(seed + T + H)
    (w1, v1), (w3, v3), (w2, v2) = experts(m, E, I, H, seed + 1), experts(m, E, I, H, seed + 2), experts(m, E, H, I, seed + 3)
    if x is None:
        x = torch.randn(T, H, generator=g) * torch.exp2(torch.randint(-4, 5, (T, 1), generator=g).float())
        x[:, torch.rand(H, generator=g) < 0.01] *= 40
        x = x.to(DT[dtype])
    if ids is None:
        ids = torch.rand(T, E, generator=g).argsort(1)[:, :k].int()
    weights = torch.rand(ids.shape, generator=g)
    y = m.sdq_mx4_moe(x.cuda(), ids.int().cuda(), weights.cuda(), w1, w3, w2, out=out, workspace=workspace)
    assert m.device_status() == 0
    xd, want, bound = x.double().cuda(), torch.zeros(T, H, dtype=torch.float64, device="cuda"), torch.zeros(T, H, dtype=torch.float64, device="cuda")
    for t in range(T):
        for j in range(ids.shape[1]):
            e = int(ids[t, j])
            if not 0 <= e < E:
                continue
            gate, up = v1[e] @ xd[t], v3[e] @ xd[t]
            h = gate * torch.sigmoid(gate) * up
            c = float(weights[t, j])
            want[t] += c * (v2[e] @ h)
            # six pieces leave at most 2^-17 of the largest magnitude of an element's block of 32 (the pieces' comment in the kernel)
            block = lambda v, n: torch.nn.functional.pad(v.abs(), (0, -n % 32)).view(-1, 32).amax(1).repeat_interleave(32)[:n]  # noqa: E731
            # gate and up: fp32 sums of exact products
            a = [v[e].abs() @ ((H * 2.0 ** -23 + 2.0 ** -21) * xd[t].abs() + 2.0 ** -17 * block(xd[t], H)) for v in (v1, v3)]
            # silu changes by at most 1.1 times its argument's change
            dh = 1.1 * a[0] * up.abs() + gate.abs() * a[1] + 1.1 * a[0] * a[1] + 2.0 ** -21 * h.abs()
            dh = dh + 2.0 ** -17 * block(h.abs() + dh, I)
            bound[t] += abs(c) * (v2[e].abs() @ dh + (I * 2.0 ** -23 + 2.0 ** -21) * (v2[e].abs() @ h.abs()))
    got = y.double()
    eps = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -11
    tol = bound * 1.01 + eps * want.abs() + 2.0 ** -24
    assert torch.isfinite(got).all()
    assert ((got - want).abs() <= tol).all(), ((got - want).abs() / tol).max().item()
    return y, want


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("T,H,I,E,k", [(1, 128, 128, 1, 1), (1, 1, 1, 2, 1), (1, 256, 384, 8, 2), (1, 2048, 1408, 16, 6), (2, 100, 33, 5, 3), (7, 520, 700, 4, 2), (16, 384, 256, 8, 4),
                                       (40, 256, 130, 3, 1), (41, 129, 257, 1, 1), (64, 260, 300, 2, 2), (64, 512, 640, 40, 8)])
def test_moe(m, dtype, T, H, I, E, k):
    check_moe(m, T, H, I, E, k, dtype)


def test_moe_is_closer_than_its_output_type(m):
    """the sums before the last rounding carry far more than its bits: nearly every output is the nearest one"""
    y, want = check_moe(m, 8, 512, 768, 4, 2, "bf16")
    assert ((y.double() - want.to(torch.bfloat16).double()).abs() > 0).double().mean() < 0.1


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_moe_ids_outside_dropped_and_twice(m, dtype):
    ids = torch.tensor([[0, 0, 0], [-1, 5, 1], [-1, -7, 6], [2, 1, 2], [99, 3, 4]])
    y, _ = check_moe(m, 5, 200, 300, 5, 3, dtype, ids=ids)
    assert (y[2] == 0).all()
    y, _ = check_moe(m, 3, 200, 300, 5, 2, dtype, ids=torch.full((3, 2), -1))
    assert (y == 0).all()


def test_moe_one_expert_for_everybody(m):
    """more pairs than one unit takes, among them a token that names an expert eight times"""
    check_moe(m, 64, 140, 150, 6, 2, "bf16", ids=torch.tensor([[3, 5]] * 63 + [[3, 3]]))
    check_moe(m, 20, 140, 150, 6, 8, "fp16", ids=torch.full((20, 8), 2))
    # (units of sixteen, for few pairs an expert in the mean)
    check_moe(m, 40, 300, 290, 32, 3, "bf16", ids=torch.tensor([[7, 31, 7]] * 25 + [[7, 0, 12]] * 15))
    check_moe(m, 64, 140, 1300, 20, 2, "bf16", ids=torch.tensor([[t % 20, 17] for t in range(64)]))


@pytest.mark.parametrize("H", [256, 250])
def test_moe_strided_tokens_outputs_and_scratch(m, H):
    (w1, _), (w3, _), (w2, _) = experts(m, 4, 96, H, 1), experts(m, 4, 96, H, 2), experts(m, 4, H, 96, 3)
    g = torch.Generator().manual_seed(3)
    big = torch.randn(12, 700, generator=g).bfloat16().cuda()
    x = big[2:9, 5:5 + H]
    ids, w = torch.randint(0, 4, (7, 2), generator=g).int().cuda(), torch.rand(7, 2, generator=g).cuda()
    want = m.sdq_mx4_moe(x.contiguous(), ids, w, w1, w3, w2)
    out = torch.full((9, H + 6), 7.0, dtype=torch.bfloat16, device="cuda")
    n = m.mx4_moe_workspace(7, 2, H, 96, "cuda").numel()
    ws = torch.full((n + 4096,), 0xFF, dtype=torch.uint8, device="cuda")          # NaN codes and scales wherever nothing is written
    y = m.sdq_mx4_moe(x, ids, w, w1, w3, w2, out=out[1:8, 3:3 + H], workspace=ws[:n])
    assert torch.equal(y, want) and (out[0] == 7).all() and (out[8] == 7).all() and (out[:, :3] == 7).all() and (out[:, 3 + H:] == 7).all()
    assert (ws[n:] == 0xFF).all()
    for _ in range(3):                                                             # the scratch of another call, larger than needed
        assert torch.equal(m.sdq_mx4_moe(x[:3], ids[:3], w[:3], w1, w3, w2, workspace=ws[:n]), want[:3])


def test_moe_a_token_that_is_not_finite_stays_alone(m):
    (w1, _), (w3, _), (w2, _) = experts(m, 3, 200, 300, 1), experts(m, 3, 200, 300, 2), experts(m, 3, 300, 200, 3)
    x = torch.randn(6, 300, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    ids, w = torch.tensor([[0, 1]] * 6).int().cuda(), torch.rand(6, 2).cuda()
    want = m.sdq_mx4_moe(x, ids, w, w1, w3, w2)
    x[1, 299], x[4, 7] = float("nan"), float("inf")
    y = m.sdq_mx4_moe(x, ids, w, w1, w3, w2)
    keep = torch.tensor([0, 2, 3, 5]).cuda()
    assert torch.isnan(y[1]).all() and torch.isnan(y[4]).all() and torch.equal(y[keep], want[keep])


def test_moe_extreme_magnitudes(m):
    """activations near both ends of bf16's range go through: pieces and their scales follow the block"""
    (w1, v1), (w3, _), (w2, _) = experts(m, 2, 128, 256, 1), experts(m, 2, 128, 256, 2), experts(m, 2, 256, 128, 3)
    x = torch.randn(4, 256, generator=torch.Generator().manual_seed(1))
    x[0] *= 2.0 ** -130
    x[1] *= 2.0 ** 60
    x[2, 1:] *= 2.0 ** -30                                                          # one large channel, the rest far below it
    x = x.bfloat16().cuda()
    y = m.sdq_mx4_moe(x, torch.zeros(4, 1).int().cuda(), torch.ones(4, 1).cuda(), w1, w3, w2)
    assert (y[0] == 0).all() and torch.isfinite(y[2:]).all() and not torch.isnan(y).all(1)[2]


def test_route_and_experts_as_a_decoder_uses_them(m):
    """router, experts and the projection behind them, captured once and replayed on other tokens; two layers at once on two streams"""
    T, H, I, E, k = 12, 512, 384, 16, 4
    g = torch.Generator().manual_seed(9)
    ws = [m.mx4_moe_workspace(T, k, H, I, "cuda") for _ in range(2)]
    (w1, v1), (w3, v3), (w2, v2) = experts(m, E, I, H, 1), experts(m, E, I, H, 2), experts(m, E, H, I, 3)
    router = (torch.randn(E, H, generator=g) / H ** 0.5).bfloat16().cuda()
    wo = m.sdq_mx4_quantize(torch.randn(H, H, generator=g).bfloat16().cuda())

    def layer(x, i, out=None):
        ids, w = m.sdq_moe_route(x, router, k)
        y = m.sdq_mx4_moe(x, ids, w, w1, w3, w2, workspace=ws[i], out=out)
        return y, m.sdq_mx4_linear(m.sdq_mx4_quantize(y), wo)

    xs = [torch.randn(T, H, generator=g).bfloat16().cuda() for _ in range(3)]
    want = [layer(x, 0) for x in xs]
    ids, w, _ = route_reference(xs[0], router, k, None, False, True)
    xd = xs[0].double()
    one = sum(float(w[3, j]) * (v2[e] @ (torch.nn.functional.silu(v1[e] @ xd[3]) * (v3[e] @ xd[3]))) for j, e in enumerate(ids[3].tolist()))
    assert ((want[0][0][3].double() - one).abs() <= 2.0 ** -7 * one.abs().max()).all()
    static = xs[0].clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        layer(static, 0)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = layer(static, 0)
    for x, y in zip(xs, want):
        static.copy_(x)
        graph.replay()
        assert torch.equal(got[0], y[0]) and torch.equal(got[1], y[1])
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = []
    for i in range(10):
        with torch.cuda.stream(streams[i % 2]):
            outs.append(layer(xs[i % 3], i % 2))
    torch.cuda.synchronize()
    assert all(torch.equal(o[0], want[i % 3][0]) and torch.equal(o[1], want[i % 3][1]) for i, o in enumerate(outs))
    assert m.device_status() == 0


def test_without_the_native_half_the_calls_go_through_ctypes(m, monkeypatch):
    """same results, same refusals, whichever half marshals"""
    T, H, I, E, k = 5, 192, 130, 6, 2
    g = torch.Generator().manual_seed(4)
    x, router = torch.randn(T, H, generator=g).bfloat16().cuda(), torch.randn(E, H, generator=g).bfloat16().cuda()
    (w1, _), (w3, _), (w2, _) = experts(m, E, I, H, 1), experts(m, E, I, H, 2), experts(m, E, H, I, 3)

    def all_calls():
        ids, w = m.sdq_moe_route(x, router, k, scale=1)
        y = m.sdq_mx4_moe(x, ids, w, w1, w3, w2)
        q = m.sdq_mx4_quantize(y, m.FMT_NVFP4)
        v = m.sdq_mx4_dequantize(q, torch.float16)
        return [ids, w, y, v, m.sdq_mx4_dequantize(w1, torch.float32), m.sdq_mx4_linear(q, q, bias=y[:, 0].contiguous()),
                m.sdq_mx4_linear(q, q, out=torch.zeros(T, T, device="cuda"))]

    def refusals():
        for bad in (lambda: m.sdq_mx4_quantize(x.int()), lambda: m.sdq_mx4_quantize(x.t()), lambda: m.sdq_mx4_quantize(x[0]), lambda: m.sdq_mx4_quantize(x, buf=x),
                    lambda: m.sdq_mx4_linear(m.sdq_mx4_quantize(x), m.sdq_mx4_quantize(x), bias=x[0]), lambda: m.sdq_mx4_quantize(x.expand(T, H).as_strided((T, H), (1, 1))),
                    lambda: m.sdq_mx4_linear(m.sdq_mx4_quantize(x), m.sdq_mx4_quantize(x), out=torch.zeros(T, T + 1, device="cuda")),
                    lambda: m.sdq_moe_route(x, router.float(), k), lambda: m.sdq_moe_route(x, router[:, 1:], k), lambda: m.sdq_moe_route(x, router, k, bias=x[0]),
                    lambda: m.sdq_mx4_moe(x, torch.zeros(T, k, device="cuda"), torch.zeros(T, k, device="cuda"), w1, w3, w2),
                    lambda: m.sdq_mx4_moe(x, torch.zeros(T, k, device="cuda").int(), torch.zeros(T, k + 1, device="cuda"), w1, w3, w2),
                    lambda: m.sdq_mx4_moe(x.cpu(), torch.zeros(T, k, device="cuda").int(), torch.zeros(T, k, device="cuda"), w1, w3, w2)):
            with pytest.raises(ValueError):
                bad()
        for bad in (lambda: m.sdq_mx4_quantize(x, 7), lambda: m.sdq_mx4_quantize(x, rule=m.SCALE_UE4M3), lambda: m.sdq_moe_route(x, router, E + 1),
                    lambda: m.sdq_mx4_linear(m.sdq_mx4_quantize(x), m.sdq_mx4_quantize(x, m.FMT_NVFP4)), lambda: m.sdq_mx4_quantize(x[:0]),
                    lambda: m.sdq_mx4_quantize(x, buf=torch.empty(1024, dtype=torch.uint8, device="cuda")),
                    lambda: m.sdq_mx4_moe(x, torch.zeros(T, k, device="cuda").int(), torch.zeros(T, k, device="cuda"), w1, w3, w1),
                    lambda: m.sdq_mx4_moe(x, torch.zeros(T, k, device="cuda").int(), torch.zeros(T, k, device="cuda"), w1, w3, w2,
                                          workspace=torch.empty(1024, dtype=torch.uint8, device="cuda"))):
            with pytest.raises(m.SdqError):
                bad()

    want = all_calls()
    refusals()
    monkeypatch.setattr(m, "_fast", m._NoNative())
    for a, b in zip(all_calls(), want):
        assert a.dtype == b.dtype and torch.equal(a, b)
    refusals()
