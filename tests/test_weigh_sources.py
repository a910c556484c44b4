"""What can only be read off the weighing kernel's source: a wait that gives up needs half a second of a copy that never ends, which no test may bring about."""
import os
import re

from paper_2601_13143_b200 import build


def _kernel(name):
    with open(os.path.join(build.CSRC, name)) as f:
        source = re.sub(r"//[^\n]*", "", f.read())
    return source[source.index("__global__"):]


def test_weights_are_stored_only_where_no_wait_gave_up():
    """Weights are added up in place, so a wrong sum cannot be taken back.  Whichever warp's wait gives up, it leaves the flag before it goes on; what came of it
    reaches the summing warps behind that.  So the flag, looked at behind the teams' barrier, keeps every sum out that may be wrong."""
    kernel = _kernel("cache_weigh_many.cu")
    stores = [m.start() for m in re.finditer(r"w\.weights\[[^\]]*\]\s*=", kernel)]
    assert len(stores) == 1
    barrier = kernel.rindex("bar.sync 1,", 0, stores[0])
    looked = re.search(r"(\w+) = \*abort == 0;", kernel[barrier:stores[0]])
    assert looked, "the flag is not looked at between the barrier and the store"
    assert re.search(r"if \([^)]*\b" + looked.group(1) + r"\b[^)]*\)\s*$", kernel[:stores[0]])


def test_a_wait_that_gives_up_leaves_the_flag_first():
    with open(os.path.join(build.CSRC, "sm100_ptx.cuh")) as f:
        source = f.read()
    wait = source[source.index("bool mbar_wait_bounded("):source.index("bool mbar_wait_warp(")]
    for m in re.finditer(r"return false;", wait):
        assert re.search(r"\*abort = 1;\s*$|if \(\*abort\) $", wait[:m.start()])
