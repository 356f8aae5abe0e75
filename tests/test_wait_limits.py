"""Waits inside kernels that have a limit: what is reported, and what is left behind, where one runs out."""
import os
import re

import paper_2310_14423_b200

CSRC = os.path.join(os.path.dirname(paper_2310_14423_b200.__file__), "csrc")


def body(source, kernel):
    """Text of a kernel's definition."""
    text = open(os.path.join(CSRC, source)).read()
    return re.search(r"\n" + kernel + r"\(.*?\n}\n", text, re.S).group(0)


def test_the_product_kernel_looks_for_waits_that_ran_out_when_all_its_warps_are_done():
    """A warp may give up after every other one has finished, so the flag is read behind the barrier that all of them reach."""
    text = body("muon.cu", "product_kernel")
    assert text.count("*p.late = 1u") == 1
    assert text.rindex("pair_sync();") < text.index("*p.late = 1u")
