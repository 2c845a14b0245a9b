"""Host side of the microscaled 4-bit operators, without a GPU: sizes, refusals, the reference's own pins."""
import ctypes

import numpy as np
import pytest
import torch

from tests import mx4_reference as ref


@pytest.fixture(scope="module")
def m():
    import paper_2406_13868_b200 as mod
    mod.build()
    return mod


def test_reference_grid_and_ties():
    assert np.array_equal(ref.e4m3_values(), torch.arange(1, 127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy())
    # boundaries: a tie goes to the even code
    codes, scales, _ = ref.quantize(np.array([[0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, -0.25, -5.0, 7.9]]), False, True)
    assert scales.tolist() == [[128]] and ref.quantize(np.array([[6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]]), False)[0].tolist() == [[7, 0, 2, 2, 4, 4, 6, 6]]
    assert codes[0, -1] == 6                                              # 3.95 -> 4


@pytest.mark.parametrize("nv", [False, True])
def test_reference_fixes_its_own_values(nv):
    """what has been quantized is quantized to itself"""
    x = np.random.default_rng(0).standard_normal((20, 77)) * 2.0 ** np.random.default_rng(1).integers(-8, 8, (20, 1))
    c, s, f = ref.quantize(x, nv)
    v = ref.values(c, s, f, nv)
    assert np.abs(v - x).max() <= np.abs(x).max() / 4
    c2, s2, f2 = ref.quantize(v, nv)
    assert np.array_equal(ref.values(c2, s2, f2, nv), v)
    assert np.array_equal(ref.unpack(ref.pack(c), 77), c)


def test_sizes(m):
    b = ctypes.c_size_t()
    L = m.lib()
    assert L.sdq_mx4_size(1, 1, 0, ctypes.byref(b)) == 0 and b.value == 17408
    assert L.sdq_mx4_size(129, 257, 1, ctypes.byref(b)) == 0 and b.value == 4 * 18432 + 1024
    assert L.sdq_mx4_size(4096, 4096, 0, ctypes.byref(b)) == 0 and b.value == 32 * 16 * 17408
    assert L.sdq_mx4_size(0, 4, 0, ctypes.byref(b)) == 2 and L.sdq_mx4_size(4, 0, 0, ctypes.byref(b)) == 2 and L.sdq_mx4_size(4, 4, 2, ctypes.byref(b)) == 1
    assert L.sdq_mx4_size(1 << 36, 1 << 30, 0, ctypes.byref(b)) == 2
    assert L.sdq_mx4_experts_size(3, 130, 200, ctypes.byref(b)) == 0 and b.value == 3 * 2 * 2 * 8704
    assert L.sdq_mx4_experts_size(0, 130, 200, ctypes.byref(b)) == 2


def test_the_abi_refuses_before_it_launches(m):
    L, d = m.lib(), m._Mx4()
    P, r = 1 << 20, ctypes.byref(d)                                       # an aligned address that nothing touches
    q = lambda *a: L.sdq_mx4_quantize(*a)  # noqa: E731
    assert q(None, 0, 4, 64, 64, 0, 0, P, 1 << 30, r, None) == 1
    assert q(P, 3, 4, 64, 64, 0, 0, P, 1 << 30, r, None) == 1
    assert q(P, 0, 4, 64, 64, 2, 0, P, 1 << 30, r, None) == 1
    assert q(P, 0, 4, 64, 64, 0, 2, P, 1 << 30, r, None) == 1
    assert q(P, 0, 4, 64, 63, 0, 0, P, 1 << 30, r, None) == 2
    assert q(P, 0, 0, 64, 64, 0, 0, P, 1 << 30, r, None) == 2
    assert q(P + 1, 0, 4, 64, 64, 0, 0, P, 1 << 30, r, None) == 3
    assert q(P, 0, 4, 64, 64, 0, 0, P + 16, 1 << 30, r, None) == 3
    assert q(P, 0, 4, 64, 64, 0, 0, P, 17407, r, None) == 5
    assert L.sdq_mx4_import(P, P, P, 4, 64, 0, P, 1 << 30, r, None) == 1   # MXFP4 has no factors
    assert L.sdq_mx4_import(P, None, None, 4, 64, 0, P, 1 << 30, r, None) == 1
    assert L.sdq_mx4_import(P, P, None, 4, 64, 0, P, 100, r, None) == 5
    assert L.sdq_mx4_experts_quantize(P, 0, 0, 4, 64, 0, P, 1 << 30, r, None) == 2
    assert L.sdq_mx4_experts_import(P, P, 2, 4, 64, P, 100, r, None) == 5
    assert L.sdq_mx4_export(r, P, P, None, None) == 1                      # an empty descriptor
    assert L.sdq_mx4_dequantize(r, P, 0, 64, None) == 1


def _desc(m, E, R, K, fmt, P=1 << 20):
    d, b = m._Mx4(), ctypes.c_size_t()
    assert (m.lib().sdq_mx4_experts_size(E, R, K, ctypes.byref(b)) if E else m.lib().sdq_mx4_size(R, K, fmt, ctypes.byref(b))) == 0
    d.dev, d.bytes, d.E, d.R, d.K, d.fmt = P, b.value, E, R, K, fmt
    n = E * -(-R // 128) * -(-K // 128) * 8704 if E else -(-R // 128) * -(-K // 256) * (18432 if fmt else 17408)
    d.factors = (n + 255) // 256 * 256
    return d


def test_the_product_refuses_operands_that_do_not_belong_together(m):
    L, P = m.lib(), 1 << 20
    x, w = _desc(m, 0, 4, 300, 0), _desc(m, 0, 200, 300, 0)
    go = lambda a, b, bias=None, dt=0, y=P, ld=200: L.sdq_mx4_linear(ctypes.byref(a), ctypes.byref(b), bias, dt, y, ld, None)  # noqa: E731
    assert go(x, _desc(m, 0, 200, 301, 0)) == 2
    assert go(x, _desc(m, 0, 200, 300, 1)) == 4
    assert go(x, _desc(m, 2, 200, 300, 0)) == 4
    assert go(x, w, ld=199) == 2
    assert go(x, w, y=P + 1) == 3 and go(x, w, y=P + 2, dt=2) == 3 and go(x, w, bias=P + 1) == 3
    assert go(x, w, y=None) == 1 and go(x, w, dt=3) == 1
    bad = _desc(m, 0, 200, 300, 0)
    bad.bytes -= 1
    assert go(x, bad) == 1
    bad = _desc(m, 0, 200, 300, 0)
    bad.R = 400                                                            # a descriptor that somebody changed
    assert go(x, bad, ld=400) == 1


def test_the_binding_refuses_what_it_cannot_pass_on(m):
    with pytest.raises(ValueError, match="CUDA"):
        m.sdq_mx4_quantize(torch.zeros(4, 64, dtype=torch.bfloat16))
    with pytest.raises(TypeError):
        m.sdq_mx4_quantize([1.0])
    with pytest.raises(ValueError, match="CUDA"):
        m.sdq_mx4_import(torch.zeros(4, 32, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.uint8))
    with pytest.raises(ValueError, match="CUDA"):
        m.sdq_mx4_experts(torch.zeros(2, 4, 64, dtype=torch.bfloat16))


def test_router_and_expert_layer_refuse_before_they_launch(m):
    L, P = m.lib(), 1 << 20
    r = lambda x=P, dt=0, T=4, H=64, ldx=64, w=P, E=8, ldw=64, bias=None, k=2, sc=0: L.sdq_moe_route(x, dt, T, H, ldx, w, E, ldw, bias, k, sc, 1, 1.0, P, P, None)  # noqa: E731
    assert r(x=None) == 1 and r(dt=3) == 1 and r(sc=2) == 1
    assert r(k=0) == 2 and r(k=9) == 2 and r(E=1025) == 2 and r(E=64, k=33) == 2 and r(T=0) == 2 and r(ldx=63) == 2 and r(ldw=63) == 2
    assert r(x=P + 1) == 3 and r(bias=P + 2) == 3
    b = ctypes.c_size_t()
    assert L.sdq_mx4_moe_workspace_size(64, 8, 4096, 11008, ctypes.byref(b)) == 0 and b.value > 0
    need = b.value
    for bad in ((65, 8, 64, 64), (0, 8, 64, 64), (1, 33, 64, 64), (1, 0, 64, 64), (1, 1, 0, 64), (1, 1, 64, 0)):
        assert L.sdq_mx4_moe_workspace_size(*bad, ctypes.byref(b)) == 2
    w1, w3, w2 = _desc(m, 8, 11008, 4096, 0), _desc(m, 8, 11008, 4096, 0), _desc(m, 8, 4096, 11008, 0)

    def go(a=w1, c=w3, d=w2, T=64, dt=0, ldx=4096, ws=P, size=need, x=P):
        return L.sdq_mx4_moe(x, dt, T, 4096, ldx, P, P, 8, ctypes.byref(a), ctypes.byref(c), ctypes.byref(d), P, 4096, ws, size, None)
    assert go(size=need - 1) == 5
    assert go(T=65) == 2 and go(ldx=4095) == 2
    assert go(dt=2) == 1 and go(x=None) == 1 and go(ws=None) == 1
    assert go(ws=P + 16) == 3 and go(x=P + 1) == 3
    assert go(a=_desc(m, 8, 11008, 4095, 0)) == 2 and go(c=_desc(m, 7, 11008, 4096, 0)) == 2 and go(d=_desc(m, 8, 4097, 11008, 0)) == 2
    assert go(a=_desc(m, 0, 11008, 4096, 0)) == 4
