"""Orders that the microscaled 4-bit kernels have to keep and that no run shows reliably, read from the sources."""
import os
import re

import pytest

from tests import test_kernel_sources as base

MX4 = os.path.join(base.CSRC, "mx4")
REMOTE = re.compile(base.REMOTE.pattern + r"|sum_over_cluster|load_cta|arrive_cta|store_to_cta")


def kernels(monkeypatch):
    monkeypatch.setattr(base, "CSRC", MX4)
    return base.kernels()


@pytest.fixture()
def bodies(monkeypatch):
    return {n: b for _, n, b in kernels(monkeypatch)}


def test_no_remote_shared_memory_before_the_cluster_has_started(bodies):
    """distributed shared memory may be touched only when all CTAs of the cluster are known to have started, and no CTA leaves before the others
    are through with its own"""
    remote = {n: b for n, b in bodies.items() if REMOTE.search(b)}
    assert {"mx4_linear_narrow_kernel", "mx4_linear_wide_kernel", "moe_route_kernel", "moe_route_mma_kernel", "moe_up_kernel", "moe_down_kernel"} <= set(remote)
    for n, b in remote.items():
        first, last = REMOTE.search(b).start(), [x.start() for x in REMOTE.finditer(b)][-1]
        syncs = [x.start() for x in re.finditer(r"ptx::cluster_sync\(\)|cluster_wait\(\)", b)]
        assert syncs[0] < first and syncs[-1] > last, n


def test_every_kernel_lets_the_next_launch_in_behind_its_own_wait(bodies):
    """a launch may read, in front of its own wait, what was complete before the launch in front of it began: the library's products read packed
    weights there, the expert layer ids and weights"""
    assert len(bodies) >= 12
    for n, b in bodies.items():
        lets_in = [x.start() for x in re.finditer(r"griddep_launch_dependents\(\)", b)]
        assert len(lets_in) == 1, n
        waits = [x.start() for x in re.finditer(r"ptx::griddep_wait\(\);", b[:lets_in[0]])]
        assert waits and "else if (warp" not in b[waits[-1]:lets_in[0]], n          # (by a thread that has waited itself)


def test_tensor_memory_is_taken_before_the_next_launch_is_let_in(bodies):
    """else the next launch could take the columns and wait for this one, which waits for them"""
    for n, b in bodies.items():
        if "tmem_alloc" in b:
            assert b.index("tmem_alloc") < b.index("griddep_launch_dependents()"), n


def test_a_products_columns_of_tensor_memory_suffice_for_what_an_sm_has_room_for():
    """256 columns come with nearly half of an SM's shared memory (1 KB of it reserved for each CTA): two leave less than any product's
    smallest ring (16 KB) takes"""
    src, moe = (open(os.path.join(MX4, n)).read() for n in ("linear.cu", "moe.cu"))
    assert "lc.dynamicSmemBytes = bytes > NARROW_LEAST ? bytes : NARROW_LEAST;" in src and "lc.dynamicSmemBytes = SMEM_MAX;" in src
    least = int(re.search(r"NARROW_LEAST = (\d+);", src).group(1))
    assert 0 < 233472 - 2 * (least + 1024) < 15000
    assert "const uint32_t room = (half ? SMEM_MAX / 2 - 1024 : SMEM_MAX) - 1024 - 128;" in moe


def test_global_memory_is_read_behind_the_wait_for_the_launch_in_front(bodies):
    """only a prefetch into L2 may come earlier: the launch in front may be the one that writes a weight matrix"""
    for n, b in bodies.items():
        if n in ("moe_up_kernel", "moe_down_kernel"):
            continue
        wait = b.index("ptx::griddep_wait()")
        for what in (r"ptx::bulk_g2s\(", r"__ldg\(", r"\bload_unit<", r"get_codes\(", r"put_codes\(", r"codes\[r", r"atomicOr\(", r"\bload8<", r"load8_raw<", r"p\.(?:ids|weights|ws)\b"):
            assert all(x.start() > wait for x in re.finditer(what, b)), (n, what)


def test_expert_layer_reads_ids_and_weights_early_only_behind_launches_that_have_waited(bodies):
    """the products read ids and expert weights in front of their own wait, which the launches in front of them, the layer's own, allow;
    the scratch, the tokens and the outputs are touched behind the wait"""
    for n in ("moe_up_kernel", "moe_down_kernel"):
        b = bodies[n]
        roles = re.split(r"\} else if \(warp", b[b.index("bool ok = true"):])
        assert sum("p.ws" in r for r in roles) == 2
        for r in roles:
            if "p.ws" in r:
                assert r.index("ptx::griddep_wait()") < r.index("p.ws")
            if "p.weights" in r:
                assert r.index("ptx::griddep_wait()") < r.index("p.weights")
    tail = bodies["moe_down_kernel"]
    assert tail.rindex("ptx::griddep_wait()") < tail.index("p.y")
