"""A commit to an mbarrier covers the products that its own thread issued, so in
the 4-bit cache's tensor-memory kernels products and commits, the ones before
tensor memory is freed among them, come from the lane that is elected for them."""
import os
import re

from tests.conftest import ROOT

SOURCE = os.path.join(ROOT, "paper_2608_15797_gb300", "csrc", "kvr_kv4_tile.cu")


def guards(text, call):
    """For every call: the headers of the blocks that it stands in."""
    text = re.sub(r"//[^\n]*", "", text)
    found, open_blocks, start = [], [], 0
    for m in re.finditer(r"[{};]|\b%s\(" % call, text):
        c = m.group()
        if c == "{":
            open_blocks.append(" ".join(text[start:m.start()].split()))
        elif c == "}":
            open_blocks.pop()
        elif c != ";":
            found.append(list(open_blocks))
            continue
        start = m.end()
    return found


def test_products_and_commits_come_from_one_lane():
    with open(SOURCE) as f:
        text = f.read()
    for call, least in (("tc_commit", 6), ("tc_mma", 1), ("tc_mma_ts", 2)):
        calls = guards(text, call)
        assert len(calls) >= least
        for blocks in calls:
            assert any(b.endswith("if (elect_one())") for b in blocks), (
                call, blocks[-3:])


def test_guards():
    text = "void f() { if (a) { g(1); } for (;;) if (elect_one()) { g(2); } }"
    assert guards(text, "g") == [["void f()", "if (a)"],
                                 ["void f()", ") if (elect_one())"]]
