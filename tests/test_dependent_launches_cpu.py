"""Kernels that start beside the end of the one before them read nothing through the read-only path: its memory must not be written while the kernel lives, and theirs
may be, until their wait is over.  No GPU needed."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2312_08728_b200", "csrc")


def functions(text):
    """Bodies of a file's functions at namespace level with what stands in front of them."""
    text = re.sub(r"//[^\n]*", "", text)
    out, depth, start = [], 0, 0
    for m in re.finditer(r"namespace[^{;]*\{|[{}]", text):
        if m.group().startswith("namespace"):
            start = m.end()
        elif m.group() == "{":
            depth += 1
        else:
            depth -= 1
            if depth <= 0:
                depth = 0
                out.append(text[start:m.end()])
                start = m.end()
    return out


def read_only(body):
    head = body[:body.index("{")]
    return bool(re.search(r"__ldg\s*\(|ld\.global\.nc", body)) or bool(re.search(r"const\s+[\w:]+\s*\*\s*__restrict__", head))


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(CSRC, "*.cuh"))), ids=os.path.basename)
def test_no_read_only_loads(path):
    found = functions(open(path).read())
    waits = [f for f in found if "wait_for_previous_kernel()" in f and "__global__" in f]
    for body in waits:
        assert not read_only(body), body[:200]
    if waits:       # (what they may call stands in the same file)
        for body in found:
            if "__global__" not in body and "{" in body:
                assert not read_only(body), body[:200]


def test_they_are_found():
    names = {re.search(r"__launch_bounds__\([^()]*\)\s*(\w+)", f).group(1) for path in glob.glob(os.path.join(CSRC, "*.cuh")) for f in functions(open(path).read())
             if "__global__" in f and "wait_for_previous_kernel()" in f}
    assert {"norm_flow_kernel", "norm_long_kernel", "norm_weight_kernel", "codes_flow_kernel", "codes_long_kernel", "int8_kernel", "int8_few_kernel", "int8_vec_kernel",
            "int8_align_kernel", "ffn_kernel", "ffn_few_kernel"} <= names, names
