"""Router: logits of any size."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def m():
    import paper_2406_13868_b200 as mod
    mod.lib()
    return mod


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
