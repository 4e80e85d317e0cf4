"""Warps that meet at a named barrier in a loop come to it for every tile, read from the kernels' sources: such a
barrier has no limit, so that a warp whose bounded wait ran out and that stayed away would leave the others
there for ever (which no run may try). It may leave the loop if it comes to the barriers that it has missed."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_26574_gb300", "csrc")


def _block(text, at):
    """The braces' content that opens first behind `at`."""
    start = text.index("{", at)
    depth = 0
    for i in range(start, len(text)):
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        if depth == 0:
            return text[start + 1:i]
    raise AssertionError("unbalanced braces")


def _loop(file, kernel):
    """The loop over key tiles of the kernel's softmax warps and what follows it, without comments."""
    with open(os.path.join(CSRC, file)) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    body = _block(text, re.search(r"\b%s\(\s*const __grid_constant__" % kernel, text).start())
    for m in re.finditer(r"for \(int j = 0; j < n_kt; \+\+j\)", body):
        loop = _block(body, m.start())
        if "red_max" in loop:
            return loop, body[body.index(loop) + len(loop) + 1:]
    raise AssertionError("no such loop")


@pytest.mark.parametrize("file,kernel", [("dard_prefix_attn.cu", "prefix_tc"), ("dard_attention.cu", "attn_tc1")])
def test_softmax_warps_miss_no_barrier(file, kernel):
    loop, behind = _loop(file, kernel)
    barrier, = re.findall(r"\w+_bar_sync\(quarter\);", loop)
    assert "bar.sync" not in loop and not re.search(r"\b(return|goto|continue)\b", loop)
    at = loop.index(barrier)
    for part, missed in ((loop[:at], "n_kt - j"), (loop[at:], "n_kt - j - 1")):
        exits = re.findall(r"missed = ([^;]*);\s*break;", part)
        assert exits and all(x == missed for x in exits)
        assert len(exits) == len(re.findall(r"\bbreak\b", part))
        # every wait's verdict is the warp's, and is looked at
        assert len(re.findall(r"\w*_wait\(&ctl", part)) == len(exits)
    assert re.match(r"\s*for \(; missed > 0; --missed\) %s" % re.escape(barrier), behind)
