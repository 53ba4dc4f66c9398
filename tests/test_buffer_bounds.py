"""Loads and stores that rely on a buffer descriptor's bounds put their whole offset where the bounds are checked (CPU).

The compiler's description of the raw buffer accesses leaves the scalar offset out of the bounds check, so it has to be
zero: an access kept in bounds by the descriptor alone would otherwise rest on what one device happens to do."""
import glob
import os
import re

from paper_2609_27193_amd.build_lib import CSRC

ACCESS = re.compile(r"__builtin_amdgcn_raw(?:_ptr)?_buffer_(load|store)_\w+\(")


def arguments(text, at):
    """The arguments of the call whose opening parenthesis ends at `at`."""
    depth, start, out = 1, at, []
    for i in range(at, len(text)):
        c = text[i]
        depth += c in "([{"
        depth -= c in ")]}"
        if depth == 0 or (depth == 1 and c == ","):
            out.append(text[start:i].strip())
            start = i + 1
        if depth == 0:
            return out
    raise AssertionError(text[at:at + 80])


def test_scalar_offsets_are_zero():
    found = 0
    for path in sorted(p for kind in ("*.hip", "*.h") for p in glob.glob(os.path.join(CSRC, kind))):
        text = open(path).read()
        for m in ACCESS.finditer(text):
            args = arguments(text, m.end())
            scalar = args[2 if m.group(1) == "load" else 3]
            assert scalar == "0", (os.path.basename(path), args)
            found += 1
    assert found >= 8
