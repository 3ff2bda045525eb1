"""Kernels start before the one in front of them in the stream has ended, whose output their inputs may
be: only a handle's own arrays, which no kernel of a call writes, go by the read-only path. Read from
the sources, since what the path returns otherwise is not defined (no GPU needed)."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2106_08846_gb300", "csrc")
# a handle's schedule, its records and its packed weights, by the names that they have in their kernels
OWN = {"spmm_dense.cu": r"(a\.table|list|a\.group_row)\b|reinterpret_cast<const uint4 \*>\(w \+|w \+", "spmm_xcol.cu": r"tab\b",
       "spmm_tcp.cu": r"(a\.trec_off|g)\b", "spmm_gk.cu": r"(a\.rec_off|grec)\b", "spmm_tc.cu": r"(a\.trec_off|trec)\b|reinterpret_cast<const int4 \*>\(trec \+"}
# what a product gets and leaves, by its parameters' names
CALLS = {"X", "bias", "ws", "Y"}


def sources():
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu")) + glob.glob(os.path.join(CSRC, "*.cuh"))):
        with open(path) as f:
            yield os.path.basename(path), re.sub(r"//[^\n]*", "", f.read())


def test_inputs_do_not_go_by_the_read_only_path():
    seen = 0
    for name, text in sources():
        assert "global.nc" not in text, name
        if name == "builder.cu":   # (launched behind the kernel before, not beside it)
            assert "launch_kernel" not in text and "pdl_" not in text
            continue
        for m in re.finditer(r"__ldg\((.{0,60})", text):
            seen += 1
            assert name in OWN and re.match(OWN[name], m.group(1)), (name, m.group(0))
    assert seen > 0


def test_no_parameter_promises_it():
    for name, text in sources():
        for m in re.finditer(r"__restrict__ (\w+)", text):
            assert m.group(1) not in CALLS, (name, m.group(1))
