"""Instructions that a warp's lanes execute together (`.sync.aligned`) come behind a
__syncwarp where lanes may have parted: read from the sources, since a kernel without
it has no defined behaviour to test (no GPU needed)."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2106_08846_gb300", "csrc")


def body(name, head):
    """The braces' contents behind the first match of `head`, without comments."""
    with open(os.path.join(CSRC, name)) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    i = text.index("{", re.search(head, text).end())
    depth, j = 1, i + 1
    while depth:
        depth += {"{": 1, "}": -1}.get(text[j], 0)
        j += 1
    return text[i + 1:j - 1].strip()


def test_a_cluster_barrier_gathers_its_warps():
    # (the lanes of k_expert_order come to it from loops of as many rounds as each lane has rows)
    assert body("ptx.cuh", r"void cluster_barrier\(\)").startswith("__syncwarp();")


def test_results_by_row_end_with_all_lanes():
    """A thread stores the rows that are the unit's: the next accumulators are loaded by whole warps."""
    put = body("fp8_product.cu", r"void put_ordered\(")
    assert put.endswith("__syncwarp();") and "return" not in put
    assert body("fp8_product.cu", r"void put\(").count("__syncwarp();") >= 4


@pytest.mark.parametrize("name,head,load", [("gated_mma.cu", r"auto load_piece = \[&\]\(.*\)", "tc5::ld_16x32"),
                                            ("spmm_dense.cu", r"for \(int gq = 0; gq < gn; gq \+= 4\)", "tc5::ld32")])
def test_accumulators_are_loaded_by_whole_warps(name, head, load):
    piece = body(name, head)
    assert 0 <= piece.find("__syncwarp();") < piece.index(load)
