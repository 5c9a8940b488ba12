"""What the sources of the FP8 and expert kernels must keep to where no run on this chip would show a lapse."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2505_14638_b200", "csrc")


def _source(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def _body(text, kernel):
    """(parameters, body) of a kernel."""
    at = re.search(r"\b%s\s*\(" % kernel, text).end()
    depth, i = 1, at
    while depth:
        depth += {"(": 1, ")": -1}.get(text[i], 0)
        i += 1
    params, start = text[at:i - 1], text.index("{", i)
    depth, j = 1, start + 1
    while depth:
        depth += {"{": 1, "}": -1}.get(text[j], 0)
        j += 1
    return params, text[start:j]


def test_the_added_rows_of_the_weighted_sum_may_be_its_result():
    # `add` may be `out`: neither is promised to be alone in its memory, nor is `add` read as memory that the kernel does not write
    params, body = _body(_source("w4a8_block_kernels.cuh"), "combine_experts_kernel")
    for name in ("add", "out"):
        decl = next(p for p in params.split(",") if re.search(r"\b%s$" % name, p.strip()))
        assert "__restrict__" not in decl, decl
    reads = re.findall(r"[\w<>]+\(add\b", body)
    assert reads == ["load8<false>(add"], reads       # (the ordinary load: __ldg is for memory that the kernel does not write)
    assert re.search(r"if constexpr \(READ_ONLY\) a = __ldg\(p\);\s*else a = \*p;", _body(_source("w4a8_block_kernels.cuh"), "load8")[1])
