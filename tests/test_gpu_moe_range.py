"""Expert layer on activations of all magnitudes, against its definition in 64 bits."""
import pytest
import torch

from tests.test_gpu_moe import experts

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.fixture(scope="module")
def m():
    import paper_2406_13868_b200 as mod
    mod.lib()
    return mod


def held(v, n):
    """what six pieces leave of a block of 32: 2^-17 of its largest magnitude, and nothing below 2^-128"""
    block = torch.nn.functional.pad(v.abs(), (0, -n % 32)).view(-1, 32).amax(1).repeat_interleave(32)[:n]
    return (2.0 ** -17 * block).clamp_min(2.0 ** -128)


def check(m, x, ids, E, I, dtype, size, seed=0):
    T, H = x.shape
    g = torch.Generator().manual_seed(seed + T)
    (w1, v1), (w3, v3), (w2, v2) = experts(m, E, I, H, seed + 1, size), experts(m, E, I, H, seed + 2, size), experts(m, E, H, I, seed + 3, size)
    x, weights = x.to(DT[dtype]), torch.rand(ids.shape, generator=g) + 0.1
    y = m.sdq_mx4_moe(x.cuda(), ids.int().cuda(), weights.cuda(), w1, w3, w2).double()
    assert m.device_status() == 0
    xd, worst = x.double().cuda(), []
    for t in range(T):
        want = torch.zeros(H, dtype=torch.float64, device="cuda")
        bound = want.clone()
        for j in range(ids.shape[1]):
            e, c = int(ids[t, j]), float(weights[t, j])
            gate, up = v1[e] @ xd[t], v3[e] @ xd[t]
            h = gate * torch.sigmoid(gate) * up
            a = [v[e].abs() @ ((H * 2.0 ** -23 + 2.0 ** -21) * xd[t].abs() + held(xd[t], H)) + 2.0 ** -148 for v in (v1, v3)]
            # silu changes by at most 1.1 times its argument's change
            dh = 1.1 * a[0] * up.abs() + gate.abs() * a[1] + 1.1 * a[0] * a[1] + 2.0 ** -21 * h.abs() + 2.0 ** -148
            dh = dh + held(h.abs() + dh, I)
            want += c * (v2[e] @ h)
            bound += c * (v2[e].abs() @ dh + (I * 2.0 ** -23 + 2.0 ** -21) * (v2[e].abs() @ h.abs()))
        eps, least = (2.0 ** -8, 2.0 ** -134) if dtype == "bf16" else (2.0 ** -11, 2.0 ** -25)
        tol = bound * 1.01 + eps * want.abs() + 2 * least
        fits = want.abs() + tol < float(torch.finfo(DT[dtype]).max)
        assert fits.any() and ((y[t] - want).abs() <= tol)[fits].all(), t
        worst.append((bound[fits] / (want.abs()[fits] + 1e-300)).median().item())
    return y, worst


@pytest.mark.parametrize("T,k", [(6, 1), (12, 2), (40, 2)])
def test_tokens_of_all_magnitudes(m, T, k):
    """hidden values from 2^-115 to 2^115, outputs that bf16 holds"""
    g = torch.Generator().manual_seed(T)
    H, I, E = 320, 290, 4
    e = torch.tensor([-56, -40, -20, 0, 20, 40, 55]).float()[torch.arange(T) % 7]
    x = torch.randn(T, H, generator=g) * torch.exp2(e)[:, None]
    y, worst = check(m, x, torch.rand(T, E, generator=g).argsort(1)[:, :k], E, I, "bf16", 0.06)
    assert (y != 0).any(1).all() and torch.isfinite(y).all()
    assert max(worst[1:6]) < 2.0 ** -3                     # (of the reference alone: the bound says something, a block with a wrong scale is off by half and more)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_blocks_of_different_magnitudes_in_a_token(m, dtype):
    g = torch.Generator().manual_seed(7)
    T, H, I, E = 20, 416, 160, 3
    wide = 30 if dtype == "bf16" else 6
    x = torch.randn(T, H, generator=g) * torch.exp2(torch.randint(-wide, wide + 1, (T, H // 32), generator=g).float()).repeat_interleave(32, 1)
    x[0] = 0
    x[0, 77] = 3.0                                         # one channel alone
    x[1, 1:] *= 2.0 ** -20                                  # one far above the rest
    x[1, 0] = 8.0
    check(m, x, torch.rand(T, E, generator=g).argsort(1)[:, :2], E, I, dtype, 0.05)


def test_the_smallest_numbers_of_fp16(m):
    g = torch.Generator().manual_seed(8)
    x = torch.randn(9, 256, generator=g) * torch.exp2(torch.arange(9).float() * 2 - 24)[:, None]
    check(m, x, torch.randint(0, 2, (9, 1), generator=g), 2, 128, "fp16", 1.0)


@pytest.mark.parametrize("T,H,I,E,k", [(1, 2048, 1408, 64, 6), (20, 500, 300, 5, 3), (64, 1024, 2048, 8, 2)])
def test_the_same_bits_every_time(m, T, H, I, E, k):
    """sums are taken in a fixed order, whatever finishes first"""
    g = torch.Generator().manual_seed(T)
    (w1, _), (w3, _), (w2, _) = experts(m, E, I, H, 1), experts(m, E, I, H, 2), experts(m, E, H, I, 3)
    x, ids, w = torch.randn(T, H, generator=g).bfloat16().cuda(), torch.randint(0, E, (T, k), generator=g).int().cuda(), torch.rand(T, k, generator=g).cuda()
    want = m.sdq_mx4_moe(x, ids, w, w1, w3, w2)
    other = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    ys = []
    for i in range(30):
        with torch.cuda.stream(other[i % 2]):
            ys.append(m.sdq_mx4_moe(x, ids, w, w1, w3, w2))
    torch.cuda.synchronize()
    assert all(torch.equal(y, want) for y in ys) and m.device_status() == 0
