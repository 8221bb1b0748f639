"""The rings of the product's kernels wait for what they read.

A stage's loads go to LDS past the registers, so the compiler cannot know when
they are needed: the kernels wait by themselves, for all but the last N loads,
counted over loads into LDS and the scales' loads into registers in the order
of their issue.  Here the code that the compiler makes is walked: at every
barrier the stage that it announces has arrived; and no loads of the two kinds
stand where the compiler may exchange them (its scheduling barriers, comments
in the listing, lie between)."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2002_09049_amd import build as hip

TILES = [(2, 1), (2, 2), (4, 2), (4, 4)]


@pytest.fixture(scope="module")
def listing(tmp_path_factory):
    assert shutil.which(hip.HIPCC), "the HIP compiler builds the library and this listing"
    out = str(tmp_path_factory.mktemp("ring") / "mx_product.s")
    subprocess.run([hip.HIPCC, *hip.FLAGS, "-I", hip.INCLUDE, "-I", hip.CSRC, "--offload-device-only", "-S",
                    os.path.join(hip.CSRC, "mx_product.hip"), "-o", out], check=True, capture_output=True)
    return open(out).read()


def ops_of(listing, symbol):
    """The kernel's loads, waits, barriers, labels and branches in order."""
    at = listing.index("\n" + symbol + ":")
    out = []
    for line in listing[at:listing.index(".Lfunc_end", at)].split("\n"):
        if "sched_barrier mask(0x00000000)" in line:
            out.append(("pin",))
        code = line.split(";")[0].strip()
        if re.match(r"(buffer|global|flat|scratch)_(load|store|atomic)", code):
            out.append(("lds",) if code.endswith(" lds") else ("other",))
        elif code.startswith("s_waitcnt"):
            m = re.search(r"vmcnt\((\d+)\)", code)
            if m:
                out.append(("wait", int(m.group(1))))
        elif code.startswith("s_barrier"):
            out.append(("barrier",))
        elif re.match(r"\.LBB\S+:", code):
            out.append(("label", code[:-1]))
        elif re.match(r"s_c?branch", code):
            out.append(("branch", code.split()[-1]))
    return out


def head_and_loop(ops):
    """Up to the loop over K, and its body."""
    where = {o[1]: i for i, o in enumerate(ops) if o[0] == "label"}
    for i, o in enumerate(ops):
        if o[0] == "branch" and where.get(o[1], len(ops)) < i and ("lds",) in ops[where[o[1]]:i]:
            return ops[:where[o[1]]], ops[where[o[1]]:i]
    raise AssertionError("no loop with loads into LDS")


def late_stages(head, loop, loads):
    """Barriers at which a load of their stage, or of an earlier one, may be in
    flight: barrier b announces stage b, load i belongs to stage i // loads."""
    flying, issued, barriers, bad = [], 0, 0, []
    for o in head + 4 * loop:
        if o[0] == "lds":
            flying.append(issued // loads)
            issued += 1
        elif o[0] == "other":
            flying.append(None)
        elif o[0] == "wait":
            flying = flying[len(flying) - o[1]:] if len(flying) > o[1] else flying
        elif o[0] == "barrier":
            stages = [s for s in flying if s is not None]
            if stages and min(stages) <= barriers:
                bad.append((barriers, flying[:]))
            barriers += 1
    assert barriers >= 16 and issued >= 16 * loads
    return bad


def mixed_regions(ops):
    """Runs of code without a scheduling barrier that hold loads of both kinds."""
    bad, kinds = 0, set()
    for o in ops:
        if o[0] in ("pin", "label", "branch", "barrier"):
            kinds = set()
        elif o[0] in ("lds", "other"):
            new = o[0] not in kinds
            kinds.add(o[0])
            bad += new and len(kinds) == 2
    return bad


KERNELS = [(f"_ZN3mpq12_GLOBAL__N_114mx_tile_kernelILi{m}ELi{n}EEEvNS_9MxProductE", m + n) for m, n in TILES]
KERNELS.append(("_ZN3mpq12_GLOBAL__N_114mx_slab_kernelENS_9MxProductE", 5))


@pytest.mark.parametrize("symbol,loads", KERNELS)
def test_stages_have_arrived(listing, symbol, loads):
    head, loop = head_and_loop(ops_of(listing, symbol))
    assert loop.count(("lds",)) == 4 * loads and loop.count(("barrier",)) == 4
    assert late_stages(head, loop, loads) == []


@pytest.mark.parametrize("symbol,loads", KERNELS)
def test_the_order_of_loads_is_fixed(listing, symbol, loads):
    head, loop = head_and_loop(ops_of(listing, symbol))
    assert mixed_regions(head) == 0 and mixed_regions(loop) == 0


def test_a_load_that_moved_is_seen(listing):
    """The walk itself: the scales' second load before those into LDS leaves one
    of stage 0's in flight."""
    head, loop = head_and_loop(ops_of(listing, KERNELS[0][0]))
    moved = list(head)
    last = max(i for i, o in enumerate(moved) if o[0] == "other")
    moved.insert(moved.index(("lds",)), moved.pop(last))
    assert late_stages(head, loop, 3) == [] and late_stages(moved, loop, 3) != []
