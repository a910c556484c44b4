"""What can only be read off the sources of the attention's kernels: an order between kernels that hardware nearly always keeps anyway."""
import os
import re

from paper_2601_13143_b200 import build


def _source(name):
    with open(os.path.join(build.CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def test_the_kernel_that_runs_beside_another_reads_behind_its_ticket():
    """attend_many_kernel beside attend_few_kernel has its own wait at its very end, and that one is for the other kernel.  What earlier work wrote it may read
    only behind the ticket which the other leaves behind its wait and ahead of its trigger, or behind a wait; index arrays never through L1."""
    few, many = _source("attend_few.cu"), _source("attend_many.cu")
    beside = few[few.index("if (c.beside)"):]
    order = [beside.index(x) for x in ("pdl_wait()", "st_release_gpu(c.ended, c.ticket)", "__syncthreads()", "pdl_trigger()")]
    assert order == sorted(order)
    kernel = many[many.index("__global__"):]
    ticket = re.search(r"if \(c\.beside && !__syncthreads_or\([^;]*ld_acquire_gpu\(c\.ended\) == c\.ticket\)\) pdl_wait\(\);", kernel)
    assert ticket and ticket.start() < kernel.index("open_list<")
    assert "chain_load_cached(" not in many
    walk = _source("attend.cuh")
    for call in re.findall(r"entry_of\(c, list, e, bad[^;]*;", walk[walk.index("open_list("):]):
        assert "through_l2" in call
    join = _source("attend.cu")
    assert re.search(r"pdl_wait\(\);\s*if \(c\.beside && [^;]*\*c\.ended = 0;", join)
