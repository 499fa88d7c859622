"""Properties of kvd_sink.hip that no run can show: read from the source."""
import os
import re

SRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2603_19664_amd", "csrc")


def calls(text, name):
    """The argument lists of the calls of builtins whose names match."""
    for m in re.finditer(name + r"\w*\(", text):
        args, depth, at = [""], 1, m.end()
        while depth:
            c = text[at]
            depth += (c in "([{") - (c in ")]}")
            if c == "," and depth == 1:
                args.append("")
            elif depth:
                args[-1] += c
            at += 1
        yield m.group(0)[:-1], [" ".join(a.split()) for a in args]


def test_row_offsets_are_range_checked():
    # Blocks of fewer than 32 keys, the empty one behind a wave's last among them, rely on the buffer's range check.
    # It covers the vector offset and the immediate; the scalar offset is outside it, or taken from the number of
    # records, which wraps where a block is shorter than that offset.
    with open(os.path.join(SRC, "kvd_sink.hip")) as f:
        found = list(calls(f.read(), r"__builtin_amdgcn_raw_(?:ptr_)?buffer_load"))
    assert len(found) >= 6
    for name, args in found:
        # (resource, LDS, size, vector offset, scalar offset, ..) and (resource, vector offset, scalar offset, ..)
        scalar = args[4 if name.endswith("_lds") else 2]
        assert scalar == "0", f"{name}({', '.join(args)})"
