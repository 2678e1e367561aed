"""The bounded waits of the 8-bit product's tensor-core kernel, read from its source: when one runs out, the kernel has to end in
order, and no call on a GPU makes one run out."""

import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_13332_b200", "csrc")


def calls(name):
    """Every call of `name` in the kernel: its text, and the headers of the blocks it stands in, outermost first."""
    text = open(os.path.join(CSRC, "stage_int8_umma.cuh")).read()
    text = re.sub(r"//[^\n]*", lambda m: " " * len(m.group()), text)
    text = text[text.index("int8_umma_kernel("):]
    found = []
    for m in re.finditer(rf"\b{name}\(", text):
        blocks, last = [], 0
        for i, c in enumerate(text[:m.start()]):
            if c == "{":
                blocks.append(" ".join(text[last:i].split()))
            elif c == "}":
                blocks.pop()
            if c in "{};":
                last = i + 1
        found.append((text[m.start():text.index("\n", m.start())], blocks))
    return found


def test_warps_give_up_as_one():
    """What a whole warp does behind a wait (tensor memory loads, warp barriers) needs all of its lanes: only single threads wait for
    themselves."""
    single = calls("mbar_wait") + calls("mbar_wait_cluster")
    assert len(single) >= 5 and len(calls("mbar_wait_warp")) == 2
    for call, blocks in single:
        assert any("lane == 0" in b for b in blocks), call
    for call, blocks in calls("mbar_wait_warp"):
        assert not any("lane == 0" in b for b in blocks), call


def test_copies_and_products_end_before_the_block():
    """Also those of a role that did not give up itself: nothing conditional on `dead` alone stands around the last waits."""
    for call, blocks in calls("mbar_wait"):
        if "drain_bar" in call or "n % S" in call:
            assert "if (dead)" not in blocks, call
