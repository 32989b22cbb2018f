"""Where the lanes of one wave exchange values through LDS without a barrier of the workgroup, the source orders it:
between a write and the next read of the same room, and between a read and the next write (no GPU needed)."""
import os
import re

import pytest

from paper_2305_04359_amd import build as B


def _body(source, head):
    """The text of the function (or lambda) whose definition begins with `head`."""
    at = source.index(head)
    first = source.index("{", at)
    depth = 0
    for i in range(first, len(source)):
        depth += {"{": 1, "}": -1}.get(source[i], 0)
        if depth == 0:
            return source[first:i + 1]
    raise AssertionError(head)


def _accesses(body):
    """'W', 'R' and '|' in their order: writes and reads of `room`, and what orders them.  Alternatives of an `if` count as
    if one followed the other."""
    out = []
    for line in body.splitlines():
        line = line.split("//")[0]
        for m in re.finditer(r"wave_exchange\(\)|(=\s*)?(?:\*reinterpret_cast<[^>]*>\(room\b[^=;]*?\)|\broom\[[^\]]*\])(\s*=(?!=))?", line):
            if m[0].startswith("wave_exchange"):
                out.append("|")
            else:
                out.append("W" if m[2] else "R")
    return "".join(out)


@pytest.mark.parametrize("name,head", [("mx_product.hip", "void store_as("), ("sample.hip", "auto sort = [&](u64 mine, u32 among)")])
def test_exchange_is_ordered(name, head):
    with open(os.path.join(B.CSRC, name)) as f:
        order = _accesses(_body(f.read(), head))
    assert "W" in order and "R" in order, order
    # (twice: the next round of a loop, or the next call, begins where this one ends)
    assert not re.search("WR|RW", order + order), order


def test_exchanges_are_all_known():
    """Every function of these files that is handed room of a wave's own is one of the above, or passes it on to one."""
    found = {}
    for name in ("mx.hip", "mx_product.hip", "mx_search.hip", "sample.hip"):
        with open(os.path.join(B.CSRC, name)) as f:
            found[name] = re.findall(r"void (\w+)\([^;{}]*\* room\)", f.read())
    assert found == {"mx.hip": [], "mx_product.hip": ["store_as", "store_results"], "mx_search.hip": [], "sample.hip": ["draw_by_wave"]}
