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
    assert {"mx4_linear_narrow_kernel", "mx4_linear_wide_kernel", "moe_route_kernel", "moe_up_kernel", "moe_down_kernel"} <= set(remote)
    for n, b in remote.items():
        first, last = REMOTE.search(b).start(), [x.start() for x in REMOTE.finditer(b)][-1]
        syncs = [x.start() for x in re.finditer(r"ptx::cluster_sync\(\)", b)]
        assert syncs[0] < first and syncs[-1] > last, n


def test_global_memory_is_read_behind_the_wait_for_the_launch_in_front(bodies):
    """every kernel lets the next launch in at once, so each waits before its first copy; only a prefetch into L2 may come earlier"""
    for n, b in bodies.items():
        wait = b.index("ptx::griddep_wait()")
        for what in (r"ptx::bulk_g2s\(", r"__ldg\(", r"\bload_unit<", r"get_codes<", r"put_codes<", r"codes\[r", r"atomicOr\(", r"\bload8<", r"load_tile\(", r"p\.(?:ids|weights|ws)\b"):
            assert all(x.start() > wait for x in re.finditer(what, b)), (n, what)
