"""The append's token lists pass between the threads of a workgroup through two buffers in LDS: tokens(x) writes the list of its block x into
buffer x % 2, request(x) reads it, barrier() separates them.  No run on a GPU shows reliably that a barrier is missing, so this reads the
order of these calls in the source, plays it for every number of blocks, and looks for accesses that no barrier separates.  Needs no GPU."""
import os
import re

import pytest

import paper_2410_12876_amd as ag

SOURCE = os.path.join(os.path.dirname(ag.LIB_PATH), "csrc", "ag_q8_fill.hip")
CALL = re.compile(r"(?:if \(([^()]*)\) )?\b(tokens|request|barrier)\(([^()]*)\);")


def calls(text):
    """[(condition, function, argument)] in the order of the text"""
    return [(m.group(1) or "True", m.group(2), m.group(3) or "0") for m in CALL.finditer(text)]


def program():
    """calls ahead of the loop over a workgroup's blocks, and those of one turn of it"""
    text = open(SOURCE).read()
    at = text.index("  if (n > 0) {\n    tokens(0);")
    loop = text.index("  for (int x = 0; x < n; ++x) {", at)
    return calls(text[at:loop]), calls(text[loop:text.index("  if (tid == 0) {  // the last workgroup that read len", loop)])


def played(n):
    """[(function, block)] of one thread of a workgroup that has n blocks"""
    ahead, turn = program()
    events = []
    for x, part in [(0, ahead)] + [(x, turn) for x in range(n)]:
        events += [(f, eval(arg, {"x": x})) for cond, f, arg in part if eval(cond, {"x": x, "n": n})]
    return events


def unseparated(events):
    """pairs of a write and a read, or of two writes, of one buffer by different blocks or threads that no barrier separates"""
    bad = []
    since = {0: [], 1: []}       # accesses of each buffer since the last barrier
    for f, x in events:
        if f == "barrier":
            since = {0: [], 1: []}
            continue
        bad += [(g, y, f, x) for g, y in since[x % 2] if "tokens" in (f, g)]
        since[x % 2].append((f, x))
    return bad


def test_the_calls_are_found():
    ahead, turn = program()
    assert [c[1] for c in ahead].count("tokens") == 2 and ("True", "request", "0") in ahead
    assert [(f, x) for c, f, x in turn if f != "barrier"] == [("request", "x + 1"), ("tokens", "x + 2")]


@pytest.mark.parametrize("n", [1, 2, 3, 4, 5, 16, 130])
def test_every_list_is_written_before_it_is_read_and_read_before_it_is_written_again(n):
    events = played(n)
    assert [x for f, x in events if f == "request"] == list(range(n)) == sorted(x for f, x in events if f == "tokens")
    assert unseparated(events) == []
