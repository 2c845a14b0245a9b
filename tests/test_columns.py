"""Tensor memory: 512 columns an SM, which nothing hands out but the allocation itself, and that waits without a limit.  So whatever thread blocks an SM has
room for, of any of the library's kernels together, must find their columns."""
import ctypes
import os
import random
import re

import pytest

import paper_2406_13868_b200 as m
from tests.test_kernel_sources import CSRC

SM, RESERVED = 233472, 1024                                    # shared memory of an SM; of it, for each thread block
i32, i64 = ctypes.c_int32, ctypes.c_int64
B200 = (ctypes.c_int(148), (ctypes.c_int * 5)(0, 0, 33, 22, 15))
CONFIGS = [m.Config(0), m.Config(1), m.Config(2), m.Config(1, 0, 32, 2), m.Config(0, m.GRAN_PAIR, 32), m.Config(0, m.GRAN_DENSE, 32), m.Config(1, m.GRAN_DENSE, 32), m.Config(2, m.GRAN_ELEM, 32)]


def linear(M, N, K, cfg, workspace=0):
    s, c = i32(), i32()
    assert m.lib().sdq_diag_linear_memory(i64(M), i64(N), i64(K), ctypes.byref(cfg), workspace, *B200, ctypes.byref(s), ctypes.byref(c)) == 0
    return s.value, c.value


def least_by_columns():
    """{columns: least shared memory} over calls of every kernel and format"""
    m.build()
    rng, least = random.Random(1), {}
    calls = [(M, N, K, cfg, ws) for M in (1, 16, 17, 32, 33, 64, 65, 128, 129, 600) for N in (128, 1024, 4096) for K in (256, 512, 2048) for cfg in CONFIGS for ws in (0, 1)]
    calls += [(int(2 ** rng.uniform(0, 12)), 128 * int(2 ** rng.uniform(0, 7)), 256 * int(2 ** rng.uniform(0, 6)), rng.choice(CONFIGS), rng.randint(0, 1)) for _ in range(3000)]
    for c in calls:
        s, cols = linear(*c)
        assert 0 < s <= SM - RESERVED
        least[cols] = min(least.get(cols, SM), s)
    for M in (1, 16, 17, 32):
        for K in range(1024, 8192, 256):
            for out_n in (0, 1):
                for x in (0, 1):
                    s, c = i32(), i32()
                    if m.lib().sdq_diag_group_memory(i64(M), i64(K), out_n, x, ctypes.byref(s), ctypes.byref(c)) == 0:
                        assert 0 < s.value <= SM - RESERVED
                        least[c.value] = min(least.get(c.value, SM), s.value)
    return least


def test_columns_suffice_for_whatever_an_sm_has_room_for():
    least = least_by_columns()
    assert set(least) == {128, 256, 512}
    # the 4-bit products and the expert layer ask for no less (the launches below go through the same function)
    sizes = {c: s + RESERVED for c, s in least.items()}
    most = [0] * (SM // RESERVED + 1)                          # columns of the thread blocks that fit into so many KB
    for kb in range(len(most)):
        for c, s in sizes.items():
            k = -(-s // RESERVED)
            if k <= kb:
                most[kb] = max(most[kb], most[kb - k] + c)
    assert max(most) <= 512


@pytest.mark.parametrize("N,K,cfg", [(1024, 2048, CONFIGS[5]), (2048, 768, CONFIGS[1]), (4096, 2048, CONFIGS[2])])
def test_calls_of_few_stages_take_their_share(N, K, cfg):
    """few tokens, K split to one to three stages a thread block: what these need, 25 to 47 KB for 128 columns, left room for four to eight of them, also
    beside thread blocks that take 256 or 512 columns"""
    m.build()
    s, c = linear(16, N, K, cfg)
    assert c == 128 and 5 * (s + RESERVED) > SM >= 4 * (s + RESERVED)
    wide, all_columns = linear(200, 384, 1536, CONFIGS[6])
    assert all_columns == 512 and wide + s + 2 * RESERVED > SM


def test_memory_queries_refuse_what_the_calls_refuse():
    m.build()
    s, c, cfg = i32(), i32(), m.Config()
    ask = lambda M, N, K: m.lib().sdq_diag_linear_memory(i64(M), i64(N), i64(K), ctypes.byref(cfg), 0, *B200, ctypes.byref(s), ctypes.byref(c))  # noqa: E731
    assert (ask(1, 128, 256), ask(0, 128, 256), ask(1, 100, 256), ask(1, 128, 200)) == (0, 2, 2, 2)
    assert m.lib().sdq_diag_linear_memory(i64(1), i64(128), i64(256), ctypes.byref(cfg), 0, *B200, None, ctypes.byref(c)) == 1
    g = lambda M, K, n, x: m.lib().sdq_diag_group_memory(i64(M), i64(K), n, x, ctypes.byref(s), ctypes.byref(c))  # noqa: E731
    assert (g(1, 1024, 1, 0), g(33, 1024, 1, 0), g(1, 768, 1, 0), g(17, 1024, 1, 1), g(1, 1024, 2, 0)) == (0, 2, 2, 2, 1)


@pytest.mark.parametrize("path", ["sdq_linear.cu", "sdq_linear_pair.cu", "sdq_linear_group.cu", "mx4/linear.cu", "mx4/moe.cu"])
def test_every_launch_that_takes_columns_asks_for_their_share(path):
    src = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, path)).read())
    assert "tmem_alloc" in src
    sizes = re.findall(r"dynamicSmemBytes = ([^;]*);", src)
    if path == "mx4/linear.cu":                                # (the wide kernel takes all there is)
        assert sizes == ["bytes > NARROW_LEAST ? bytes : NARROW_LEAST", "SMEM_MAX"]
        assert "static_assert(NARROW_LEAST == shared_for_columns(0, 256) && SMEM_MAX >= shared_for_columns(0, 512));" in src
    elif path == "mx4/moe.cu":
        launches = re.findall(r"Launch l\((.*), stream\);", src)
        assert len(launches) == 3 and sum("shared_for_columns(" in x and "p.tmem_cols)" in x for x in launches) == 2
    else:
        assert len(re.findall(r"return \(int\)shared_for_columns|return shared_for_columns|= shared_for_columns", src)) >= 1
        real = {"few_shared(p)", "shared_for_columns((size_t)p.ring_bytes + PAIR_TAIL, 512)", "(size_t)smem"}
        assert all(x in real or x == "200 * 1024" for x in sizes)          # (200 KB: an occupancy query, nothing is launched)
        if "(size_t)smem" in sizes:
            assert "const int smem = group_shared(" in src


def test_nothing_else_takes_columns():
    files = []
    for d, _, names in os.walk(CSRC):
        files += [os.path.relpath(os.path.join(d, n), CSRC) for n in names if n.endswith(".cu") and "tmem_alloc" in open(os.path.join(d, n)).read()]
    assert sorted(files) == ["mx4/linear.cu", "mx4/moe.cu", "sdq_linear.cu", "sdq_linear_group.cu", "sdq_linear_pair.cu"]
