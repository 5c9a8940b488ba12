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


def test_registers_are_redistributed_by_whole_groups_of_four_warps():
    # setmaxnreg is defined only where all warps of a group of four run the same instruction: one for warps 8 to 11 and one for 0 to 7,
    # each ahead of the branches by role, and none elsewhere
    for name in sorted(os.listdir(CSRC)):
        if name.endswith((".cu", ".cuh")) and name != "w4a8_linear_blocks.cuh":
            assert "setmaxnreg" not in _source(name), name
    text = _source("w4a8_linear_blocks.cuh")
    body = _body(text, "linear_blocks_wide_kernel")[1]
    assert text.count("setmaxnreg") == body.count("setmaxnreg") == 2
    low = re.search(r'if \(warp >= 8\) \{\s*asm volatile\("setmaxnreg\.dec\.sync\.aligned\.u32 (\d+);"\);', body)
    high = re.search(r'\n    \} else \{\s*asm volatile\("setmaxnreg\.inc\.sync\.aligned\.u32 (\d+);"\);', body)
    assert low and high and low.start() < high.start()
    # what is given out is what the block was launched with, 168 registers a thread (65536 over 384 threads, in eights)
    assert int(low.group(1)) * 128 + int(high.group(1)) * 256 <= 65536 // 384 // 8 * 8 * 384
