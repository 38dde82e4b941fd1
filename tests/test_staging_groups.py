"""Staging of the integer product's epilogue: a unit is filled again once the copies out of it have been read.  The wait counts groups of copies, so every unit has to
leave one behind, whichever way it went out: a launch may hold a product that tensor copies store and one that they cannot, and a warp's units then alternate between
the two.  No run shows a missing group reliably, the source does."""
import itertools
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2105_13890_b200", "csrc")


def block(text, at):
    """From the brace at or behind `at` to its partner."""
    start = text.index("{", at)
    depth = 0
    for i in range(start, len(text)):
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        if depth == 0:
            return text[start:i + 1], i + 1
    raise AssertionError("braces do not match")


def groups():
    """-> groups that a unit leaves behind when tensor copies store it, and when they do not."""
    with open(os.path.join(CSRC, "eoq_lin_gemm.cu")) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    chunk, _ = block(text, text.index("void write_chunk("))
    body, _ = block(chunk, chunk.index("auto out ="))
    by_copy, end = block(body, body.index("if (a.tensor_store)"))
    assert body[end:].lstrip().startswith("else")
    by_rows, end = block(body, end)
    assert body.count("++units") == 1 and body.count("store_commit()") == by_copy.count("store_commit()") + by_rows.count("store_commit()")
    return {True: by_copy.count("store_commit()"), False: by_rows.count("store_commit()")}


@pytest.mark.parametrize("units", [1, 2])
def test_a_unit_is_not_filled_while_it_is_read(units):
    left = groups()
    for way in itertools.product((True, False), repeat=6):
        order, last = [], {}          # the groups in their order: the unit that they read, or none; of a unit: the last copy out of it
        for k, copied in enumerate(way):
            unit = k % units
            done = max(0, len(order) - (units - 1))          # all but the units - 1 newest are waited for
            assert last.get(unit, -1) < done, "unit %d filled while a copy reads it: %s" % (unit, way)
            for _ in range(left[copied]):
                order.append(unit if copied else None)
            if copied:
                last[unit] = len(order) - 1
