"""Router: every token and place for itself against the definition in 64 bits, up to the numbers of tokens of a prompt, and logits of any size."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def m():
    import paper_2406_13868_b200 as mod
    mod.lib()
    return mod


def check_route(m, x, w, k, bias, sigmoid, renorm, scale=1.0):
    ids, weights = m.sdq_moe_route(x.cuda(), w.cuda(), k, bias=None if bias is None else bias.cuda(), scoring=m.ROUTE_SIGMOID if sigmoid else m.ROUTE_SOFTMAX,
                                   renorm=renorm, scale=scale)
    assert m.device_status() == 0
    ids, weights = ids.cpu().long(), weights.cpu().double()
    T, E = x.shape[0], w.shape[0]
    logits, mag = x.double() @ w.double().T, x.double().abs() @ w.double().abs().T
    # A logit's fp32 part: 16-bit operands, 32 exact products on the tensor core, which may cut what it adds, less than a unit of the running sum each;
    # fp32 operands, eight rounded multiplications and additions in one operation each.  The 64-bit sums behind them count for nothing
    err = (8 * 2.0 ** -24 if x.dtype == torch.float32 else 32 * 2.0 ** -23) * mag
    if sigmoid:
        score = torch.sigmoid(logits)
        e = torch.maximum(torch.sigmoid(logits + err) - score, score - torch.sigmoid(logits - err)) + 2.0 ** -50
    else:
        # its own logit and the sum of all: a factor within exp(+-2 max err)
        score = torch.softmax(logits, 1)
        e = score * torch.expm1(2 * err.max(1, keepdim=True)[0]) + 2.0 ** -50 * score
    choice = score if bias is None else score + bias.double()
    e = e + 2.0 ** -50 * choice.abs()
    assert ((ids >= 0) & (ids < E)).all() and (torch.sort(ids, 1)[0].diff(dim=1) > 0).all()
    # the chosen of place j is within the errors of the j-th largest
    mine, mine_e = choice.gather(1, ids), e.gather(1, ids)
    least, most = (torch.sort(c, 1, descending=True)[0][:, :k] for c in (choice - e, choice + e))
    assert (mine + mine_e >= least).all() and (mine - mine_e <= most).all()
    # and is the reference's wherever nobody else is as near: behind all in front of it, in front of all behind it
    order = torch.sort(choice, dim=1, descending=True, stable=True)[1]
    low, high = (choice - e).gather(1, order), (choice + e).gather(1, order)
    front = torch.cat([torch.full((T, 1), float("inf"), dtype=torch.float64), torch.cummin(low, 1)[0][:, :-1]], 1)
    back = torch.cat([torch.flip(torch.cummax(torch.flip(high, [1]), 1)[0], [1])[:, 1:], torch.full((T, 1), -float("inf"), dtype=torch.float64)], 1)
    sure = ((high < front) & (low > back))[:, :k]
    assert (ids == order[:, :k])[sure].all()
    p = score.gather(1, ids)
    rel = (e.gather(1, ids) / p.clamp_min(1e-300)).max(1, keepdim=True)[0]
    want = (p / p.sum(1, keepdim=True) if renorm else p) * scale
    # (normalised: the chosen's errors and their sum's; two roundings to fp32, of `scale` and of the result)
    assert ((weights - want).abs() <= (2.01 * rel + 2.0 ** -23) * want.abs() + 2.0 ** -149).all()
    return sure.double().mean().item()


@pytest.mark.parametrize("sigmoid,bias,renorm", [(False, False, True), (False, True, False), (True, False, False), (True, True, True)])
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("T,H,E,k", [(3, 4096, 128, 8), (64, 1024, 256, 8), (64, 1030, 257, 9), (5, 64, 1024, 32), (2, 2048, 1000, 17), (7, 96, 129, 1), (700, 128, 64, 6), (2051, 512, 256, 8),
                                     (1025, 77, 40, 4)])
def test_route_token_by_token(m, sigmoid, bias, renorm, dtype, T, H, E, k):
    g = torch.Generator().manual_seed(T + 3 * H + E)
    x = torch.randn(T, H, generator=g).to(DT[dtype])
    w = (torch.randn(E, H, generator=g) / H ** 0.5).to(DT[dtype])
    b = 0.1 * torch.randn(E, generator=g) if bias else None
    sure = check_route(m, x, w, k, b, sigmoid, renorm, 2.5)
    assert sure > 0.5                                  # (most places have one answer)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("E", [16, 200])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("e", [20, 31, 36, 44, 60, 100, 126])
def test_softmax_of_logits_that_fp32_holds_coarsely(m, dtype, E, bias, e):
    """logits about 2^e that differ in bits fp32 does not have: relative to the largest one in fp32 they would be off by far more than exp takes"""
    T, H = 6, 64
    g = torch.Generator().manual_seed(e)
    # two channels in different 64-bit sums: 2^e times a few for all experts alike, and to each expert up to seven quarters of half a unit of that in fp32
    x, w = torch.zeros(T, H), torch.zeros(E, H)
    x[:, 0], w[:, 0] = torch.tensor([1.0, 1.5, -1.0, 3.0, -1.25, 0.0]), 2.0 ** e
    x[:, 40], w[:, 40] = 1.0, torch.randint(0, 8, (E,), generator=g).float() * 2.0 ** (e - 26)
    x, w = x.to(DT[dtype]), w.to(DT[dtype])
    b = torch.linspace(0, 1e-3, E) if bias else None
    ids, weights = m.sdq_moe_route(x.cuda(), w.cuda(), 4, bias=None if b is None else b.cuda())
    logits = x.double() @ w.double().T                 # (exact: 28 bits)
    score = torch.softmax(logits, 1)
    choice = score if b is None else score + b.double()
    order = torch.sort(choice, dim=1, descending=True, stable=True)[1][:, :4]
    p = score.gather(1, order)
    assert torch.isfinite(weights).all()
    assert torch.equal(ids.cpu().long(), order)
    assert ((weights.cpu().double() - p / p.sum(1, keepdim=True)).abs() <= 2.0 ** -22).all()
