"""The softmax groups of gvote_attend8 meet at named barriers that have no time limit: every warp of a group has to reach each
of them, also when a bounded wait ran out for some of its warps and not for others.  So whether a barrier is reached may hang
on the walk over the tiles (the same for all warps) and on what a barrier returned, and on nothing that a warp reads after a
wait that may have failed.  Checked on the source, since a wait that runs out cannot be made on purpose.  CPU only."""
import os
import re

import pytest

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2509_03136_b200", "csrc", "attend8.cu")
# the walk and what the code computes from it alone, constants of the launch
UNIFORM = {"at", "s0", "s1", "t", "first", "kTurns", "kRb", "kR", "kBoxes", "L", "a", "max_q", "group_any", "bar_id", "g", "i", "k",
           "int", "const", "done", "next_segment"}


def softmax_role(text):
    begin = text.index("softmax: thread = row of the tile")
    end = text.index("// Running (maximum, sum relative to it)")
    body = re.sub(r"//[^\n]*", "", text[begin:end])
    return body[:body.index("atomicExch")]


def guards_of(body, call):
    """For every place of `call`, the headers of the blocks around it (if (...), for (...), else, plain)."""
    stack, found, start = [], [], 0
    for m in re.finditer(r"[{};]|%s\(" % call, body):
        if m.group() == "{":
            stack.append(body[start:m.start()].strip())
        elif m.group() == "}":
            if stack:
                stack.pop()
        elif m.group() != ";":
            found.append((m.start(), list(stack), body[start:m.start()].strip()))
            continue
        # the parts of a for header are no statements
        if body[start:m.start()].count("(") == body[start:m.start()].count(")"):
            start = m.end()
    return found


def names(header, call_results):
    header = re.sub(r"group_any\([^()]*\)", "group_any", header)          # what a barrier returns is the same for all
    header = re.sub(r"\.\w+", "", header)                                  # a member goes by what it is a member of
    return set(re.findall(r"[A-Za-z_]\w*", header)) - call_results


def test_named_barriers_hang_on_nothing_that_a_failed_wait_leaves_open():
    body = softmax_role(open(SOURCE).read())
    found = guards_of(body, "group_any")
    assert len(found) >= 5
    for at, headers, before in found:
        for h in headers + [before]:
            if not re.match(r"(else\s*)?(if|for|while)\b", h):
                # a barrier in an expression must not be skipped by what stands before it
                assert "&&" not in h and "||" not in h and "?" not in h or h in headers, h
                continue
            inside = names(re.sub(r"^(else\s*)?(if|for|while)", "", h), set())
            assert inside <= UNIFORM, f"a barrier hangs on {sorted(inside - UNIFORM)}: {h}"


@pytest.mark.parametrize("bad", ["if (rb == 0 && x.nq > 1) { group_any(bar_id, false); }", "if (ok) { group_any(bar_id, over); }",
                                 "ok = ok && group_any(bar_id, over);"])
def test_the_check_itself(bad):
    found = guards_of(bad, "group_any")
    (_, headers, before), = found
    hangs = any(names(re.sub(r"^(if|for)", "", h), set()) - UNIFORM for h in headers) or "&&" in before
    assert hangs
