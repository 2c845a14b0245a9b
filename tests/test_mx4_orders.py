"""Orders of the microscaled 4-bit kernels, read from the sources by what each role of a kernel does."""
import os
import re

import pytest

from tests.test_mx4_sources import MX4, kernels


@pytest.fixture()
def bodies(monkeypatch):
    return {n: b for _, n, b in kernels(monkeypatch)}


def roles(body):
    """the branches of the first chain over the warp's number: condition -> code, comments aside"""
    at = re.compile(r"if \(warp == 0[^{]*\) \{").search(body, body.index("bool ok = true;")).start()
    out = {}
    while True:
        cond = re.compile(r"(?:else )?if \((warp[^{]*)\) \{").match(body, at)
        if not cond:
            return out
        depth, end = 1, cond.end()
        while depth:
            depth += {"{": 1, "}": -1}.get(body[end], 0)
            end += 1
        out[cond.group(1)] = body[cond.end():end]
        at = end + (1 if body[end] == " " else 0)


def test_the_odd_cta_s_operands_are_passed_on_with_release(bodies):
    """the thread that issues a pair's MMAs learns that the other CTA's copies have landed from a thread that has waited for them, through an operation that releases at
    cluster scope, and acquires at that scope; arrivals without release carry nothing of shared memory and come on top"""
    parts = roles(bodies["mx4_linear_wide_kernel"])
    issuer = parts["warp == 1"]
    waits = re.findall(r"mbar_wait_cluster\(&(\w+)\[", issuer)
    assert len(waits) == 1 and issuer.index("mbar_wait_cluster") < issuer.index("ptx::mma2_")          # (acquire at cluster scope, for every stage)
    bar = waits[0]
    tells = [r for r in parts.values() if "st_async" in r or re.search(r"arrive\.release\.cluster", r)]
    assert len(tells) == 1
    tell = tells[0]
    assert "ptx::mapa_u32(ptx::smem_u32(%s), 0)" % bar in tell and "mbar_expect_tx(&%s[" % bar in tell     # (that very barrier, in the leader)
    assert tell.index("wait32(at_slot.full, at_slot.ph)") < tell.index("mbar_wait(&empty[") < tell.index("mbar_expect_tx") and tell.index("mbar_wait(&empty[") < tell.rindex("st_async")
    # whoever arrives there is counted: the scales' four warps of both CTAs, and the leader's expectation of the odd CTA's word
    scales = [r for r in parts.values() if "arrive_leader(&%s[" % bar in r]
    assert len(scales) == 1 and "mbar_init(&%s[i], 9)" % bar in bodies["mx4_linear_wide_kernel"]
    assert scales[0].index("tmem_st_wait") < scales[0].index("tc_fence_before") < scales[0].index("arrive_leader")


def test_a_streaming_quantizer_whose_wait_gives_up_leaves_as_a_whole(bodies):
    """whether a wait gave up is decided for the thread block, at a barrier that all warps reach; its flag is set whichever lane saw it, and
    the copies under way into its shared memory are waited for"""
    b = bodies["nv4_quantize_stream_kernel"]
    wait = re.search(r"const bool (\w+) = __all_sync\(0xffffffffu, wait32\(ptx::smem_u32\(&full\[n\]\), ph\)\);", b)
    assert wait
    left = b[b.index("if (!__syncthreads_and(%s))" % wait.group(1)):]
    depth, end = 0, left.index("{")
    while True:
        depth += {"{": 1, "}": -1}.get(left[end], 0)
        end += 1
        if not depth:
            break
    gone = left[:end]
    assert gone.index("atomicOr(&flags[FLAG_TIMEOUT], 1u)") < gone.index("wait32(") < gone.index("return;")
    assert len(re.findall(r"\breturn;", b)) == 1 and b.count("wait32(") == 2          # (no other way out)


@pytest.mark.parametrize("kernel,role,by", [("mx4_linear_narrow_kernel", "warp == 1", "at"), ("mx4_linear_wide_kernel", "warp == 2", "at_slot"), ("moe_up_kernel", "warp == 1", "at"),
                                            ("moe_down_kernel", "warp == 1", "at")])
def test_a_thread_block_whose_wait_gives_up_waits_for_its_copies(bodies, kernel, role, by):
    """the thread that empties the ring, in order, waits with a limit for what may still be under way; the barriers at the kernel's end lie behind it"""
    body = bodies[kernel]
    part = roles(body)[role]
    assert re.search(r"\{ atomicOr\(&p\.flags\[FLAG_TIMEOUT\], 1u\); wait_for_copies\(%s, (NSLOT|WIDE_SLOTS)\); \}" % by, part)
    assert re.search(r"wait32\(%s\.full, %s\.ph\)" % (by, by), part)
    tail = body[body.index(part) + len(part):]
    assert re.search(r"cluster_sync\(\)|__syncthreads\(\)", tail)


@pytest.mark.parametrize("kernel", ["mx4_linear_narrow_kernel", "mx4_linear_wide_kernel", "moe_up_kernel", "moe_down_kernel"])
def test_every_role_that_waits_reports_a_wait_that_gave_up(bodies, kernel):
    """each of them, the epilogues too: the wait that gave up may be the only one"""
    for cond, part in roles(bodies[kernel]).items():
        if re.search(r"mbar_wait|wait32", part):
            assert "atomicOr(&p.flags[FLAG_TIMEOUT], 1u)" in part, cond
        elif "produce(" in part:
            assert "p.flags" in part, cond


READS = {                              # what reads global memory through more than a plain subscript -> kernels that do so
    r"\bload16<": {"mx4_quantize_kernel", "nv4_quantize_kernel"},
    r"(?<!auto )\bload\(": {"nv4_quantize_stream_kernel"},
    r"\bcopy32\(": {"mx4_linear_narrow_kernel"},
    r"\bbulk_g2s\(": {"mx4_linear_wide_kernel"},
    r"\bget_codes\(": {"mx4_export_kernel", "mx4_dequantize_kernel"},
    r"\bcodes\[r \* kb": {"mx4_import_kernel", "mx4_export_kernel"},
    r"\bload8<": {"moe_route_kernel"},
    r"\bload8_raw<": {"moe_route_mma_kernel"},
    r"reinterpret_cast<const T\*>\(p\.x\)": {"moe_split_kernel"},
}


@pytest.mark.parametrize("what", list(READS))
def test_reads_of_global_memory_lie_behind_the_wait(bodies, what):
    """every kernel that reads so does it behind its wait for the launch in front (the expert layer's two products, which read what is complete before, aside)"""
    found = set()
    for n, b in bodies.items():
        if n in ("moe_up_kernel", "moe_down_kernel"):
            continue
        if n == "nv4_quantize_stream_kernel" and "copy32" in what:
            # (inside the function that the row before looks for the calls of)
            load = b.index("auto load = [&]")
            assert all(load < x.start() < b.index("};", load) for x in re.finditer(what, b))
            continue
        at = [x.start() for x in re.finditer(what, b)]
        if at:
            found.add(n)
            assert min(at) > b.index("ptx::griddep_wait()"), n
    assert found == READS[what]


def test_every_kernel_that_is_given_operands_is_among_them(bodies):
    assert set().union(*READS.values()) | {"moe_up_kernel", "moe_down_kernel"} == set(bodies)


def test_row_maxima_are_exchanged_between_two_cluster_barriers(bodies):
    """peers' shared memory is written when all of them have started, and read when all of them have written"""
    src = re.sub(r"//[^\n]*", "", open(os.path.join(MX4, "quant.cu")).read())
    at = src.index("__device__ __forceinline__ float max_over_cluster(")
    body = src[src.index("{", at):src.index("\n}\n", at)]
    alone, rest = body.split("if (ctas == 1) {", 1)
    assert "cluster" not in alone and "return a;" in rest[:rest.index("}")]
    remote = [x.start() for x in re.finditer(r"st\.shared::cluster", rest)]
    syncs = [x.start() for x in re.finditer(r"ptx::cluster_sync\(\)", rest)]
    assert len(syncs) == 2 and remote and syncs[0] < min(remote) <= max(remote) < syncs[1] < rest.index("m.cta[c][")
    assert [n for n, b in bodies.items() if "max_over_cluster(" in b] == ["nv4_quantize_kernel"]
