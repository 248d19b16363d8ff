"""Loads through buffers in the 8-bit products and in attention over packed prompts leave rows and steps
past the end to the buffer's range check.  That check is sure of the vector offset only (a scalar offset
counts towards the address, but a check may leave it out, or wrap where it alone lies past the end): so the
scalar offset of every such load is 0."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_14586_amd", "csrc")
LOADS = {"__builtin_amdgcn_raw_buffer_load_b32": 2, "__builtin_amdgcn_raw_buffer_load_b128": 2,
         "__builtin_amdgcn_raw_ptr_buffer_load_lds": 4}  # argument that is the scalar offset


def _arguments(text, at):
    """Of the call whose opening bracket is at `at`."""
    depth, args = 0, [""]
    for c in text[at:]:
        depth += c in "([{"
        depth -= c in ")]}"
        if depth == 0:
            return [a.strip() for a in args]
        if c == "," and depth == 1:
            args.append("")
        elif not (depth == 1 and c == "(" and args == [""]):
            args[-1] += c


@pytest.mark.parametrize("name,least", [("w8.hip", 5), ("attention_packed.hip", 1)])
def test_no_scalar_offset_decides_a_range(name, least):
    with open(os.path.join(CSRC, name)) as f:
        text = re.sub(r"//.*", "", f.read())
    calls = [(m.group(), _arguments(text, m.end())) for m in re.finditer(r"__builtin_amdgcn_raw_(?:ptr_)?buffer_load\w+", text)]
    assert len(calls) >= least and all(builtin in LOADS for builtin, _ in calls)
    assert [a for builtin, a in calls if a[LOADS[builtin]] != "0"] == []
