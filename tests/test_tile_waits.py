"""The tile products' warps read tensor memory and meet at barriers as whole
warps (the .sync.aligned forms).  A bounded wait can give up in one lane and
succeed in another, so every wait's outcome has to be agreed on by its warp."""
import os
import re

from paper_2012_11346_gb300 import build


def test_every_wait_of_the_tile_products_is_the_warps():
    text = open(os.path.join(build.CSRC, "lm_gemm.cuh")).read()
    text = re.sub(r"//[^\n]*", "", text)
    waits = [m.start() for m in re.finditer(r"\bmbar_wait\(", text)]
    assert waits
    for at in waits:
        before = re.split(r"[;{}]", text[:at])[-1]
        assert re.search(r"__all_sync\(\s*0xffffffffu\s*,\s*tc::$", before), before
