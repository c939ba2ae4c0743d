"""The sums over a row's threads of the norms between two blocks, as a model on the CPU: what a warp writes to shared memory for one sum
must not meet what another still reads for an earlier one.

A sum is: every warp writes its part to a slot, all meet, every warp reads all parts of the slot.  A warp that is ahead may be anywhere up
to the next meeting while one that is behind still reads, so of two accesses to a slot by different warps, one of them a write,
a meeting has to lie between.  Which slots the calls take is read from the kernels' source."""
import os
import re

import pytest

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2307_14995_b200", "csrc", "la_block_norm_kernels.cuh")


def body(start, end):
    text = re.sub(r"//[^\n]*", "", open(SOURCE).read())
    at = text.index(start)
    return text[at:text.index(end, at)]


def slots_named(kernel, end):
    """The slots that the calls of a direct kernel name, in the order of its source."""
    return re.findall(r"\bsum\(\w+, (\d), \w+\)", body("void __launch_bounds__(LANES%s) %s(" % (" > THREADS ? LANES : THREADS" if "fwd" in kernel else "", kernel), end))


def overlaps(ops):
    """ops: the sums' slots in order, "meet" for a barrier besides theirs.  Slots written while they may be read."""
    at, found = 0, []  # at: meetings so far
    read = {}          # slot -> the last interval between meetings in which it was read
    for op in ops:
        if op == "meet":
            at += 1
            continue
        if read.get(op) == at:
            found.append(op)
        at += 1
        read[op] = at
    return found


FORWARD = ("block_norm_fwd_kernel", "template <typename T, typename TR, int LANES, int NV, bool VEC>")
BACKWARD = ("block_norm_bwd_kernel", "struct RingRow")


@pytest.mark.parametrize("rows", [1, 2, 3, 10])
@pytest.mark.parametrize("post_norm", [True, False])
@pytest.mark.parametrize("want_n", [True, False])
def test_forward(rows, post_norm, want_n):
    of_y, of_h = slots_named(*FORWARD)
    text = body("block_norm_fwd_kernel(", FORWARD[1])
    meets = "alternate = a.post_norm && a.n;" in text and re.search(r"if \(!alternate\) __syncthreads\(\);\s*if \(!a\.n\) continue;", text) is not None
    between = ["meet"] if meets and not (post_norm and want_n) else []
    assert overlaps(([of_y] * post_norm + between + [of_h] * want_n) * rows) == []


@pytest.mark.parametrize("rows", [1, 2, 3, 10])
@pytest.mark.parametrize("post_norm", [True, False])
@pytest.mark.parametrize("dn", [True, False])
def test_backward(rows, post_norm, dn):
    of_y, of_h, of_dot, of_p = slots_named(*BACKWARD)
    meets = re.search(r"__syncthreads\(\);\s*\}\s*float\* const part", body("block_norm_bwd_kernel(", BACKWARD[1])) is not None
    assert overlaps(([of_y] * post_norm + [of_h, of_dot] * dn + [of_p] * post_norm + ["meet"] * meets) * rows) == []


def test_a_slot_of_its_own_for_every_sum_would_be_met():
    """The model finds the fault: slots by what is summed up, where a row has one sum only."""
    assert overlaps(["0", "1"] * 5) == [] and overlaps(["1"] * 5) != []
