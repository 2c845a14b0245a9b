"""How the microscaled 4-bit calls are laid out on an SM, from the functions that decide it; no GPU."""
import ctypes
import random

import pytest

import paper_2406_13868_b200 as m

i32, i64 = ctypes.c_int32, ctypes.c_int64
SHARED = 227328                       # bytes a thread block can ask for beside what the kernel has of its own


def rows(R, K, ld=None, dtype=0, address=1 << 20):
    m.build()
    r, b, s = i32(-1), i32(-1), i64(-1)
    st = m.lib().sdq_diag_mx4_quantize_rows(ctypes.c_uint64(address), i64(R), i64(K), i64(K if ld is None else ld), i32(dtype), ctypes.byref(r), ctypes.byref(b), ctypes.byref(s))
    assert st == 0
    return r.value, b.value, s.value


def test_which_rows_are_streamed():
    assert rows(8192, 11008) == (4, 2, 8 * 22016) and rows(515, 8200) == (4, 3, 12 * 16400)
    assert rows(400, 12000, 12008, 1) == (4, 2, 8 * 24000) and rows(261, 16400) == (2, 3, 6 * 32800) and rows(200, 24576, 24592) == (2, 2, 4 * 49152)
    assert rows(4, 11008) == rows(8192, 8192) == rows(8192, 11008, dtype=2) == rows(8192, 11009) == rows(8192, 11008, 11012) == rows(8192, 11008, address=8) == (0, 0, 0)
    assert rows(100, 28416)[0] == 0 and rows(148, 28416) == (2, 2, 4 * 56832) and rows(1000, 28424) == (0, 0, 0)


@pytest.mark.parametrize("K", [1 << 29, (1 << 29) + 8, (1 << 29) + 3500 * 4, (1 << 30) - 8, 1 << 30])
@pytest.mark.parametrize("dtype", [0, 1])
def test_rows_of_a_gigabyte_are_not_streamed(K, dtype):
    """their bytes, times four, pass 32 bits: two buffers of them do not fit"""
    for R in (1, 5, 1 << 10):
        assert rows(R, K, dtype=dtype) == (0, 0, 0)


def test_buffers_fit_wherever_rows_are_streamed():
    rng = random.Random(3)
    streamed = 0
    for _ in range(20000):
        K, R = 8 * int(2 ** rng.uniform(0, 27)), int(2 ** rng.uniform(0, 30))
        if (K + 127) // 128 * ((R + 127) // 128) > 1 << 40:
            continue
        r, b, s = rows(R, K, dtype=rng.randint(0, 1))
        streamed += r > 0
        assert r in (0, 2, 4) and s == r * b * 2 * K <= SHARED and (r == 0 or 2 <= b <= 8) and (r == 0 or R * K >= 1 << 22)
    assert streamed > 100
