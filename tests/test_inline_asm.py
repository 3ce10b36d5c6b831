"""Inline assembly in the kernel sources.  The compiler keeps the distances that the hardware asks for (a vector instruction
behind the matrix instruction whose result it reads, for one) between its own instructions; it does not look into assembly
text.  So the only instructions written that way are the loads from global memory straight into LDS, whose operands are
addresses; every other block is empty and only pins a value to its place."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2506_15545_amd", "csrc")
LDS_LOAD = re.compile(r"s_mov_b32 m0, %\d; s_nop \d; global_load_lds_dwordx4 %0, (off|%1)")


def test_inline_assembly_holds_nothing_but_loads_into_lds():
    texts = []
    for path in sorted(glob.glob(os.path.join(CSRC, "*.h*p"))):
        for m in re.finditer(r'\basm\s+volatile\s*\(\s*"([^"]*)"', re.sub(r"//[^\n]*", "", open(path).read())):
            texts.append((os.path.basename(path), m.group(1).replace("\\n\\t", "; ")))
    assert sum(bool(t) for _, t in texts) == 2    # the two forms of the load
    for name, text in texts:
        assert not text or LDS_LOAD.fullmatch(text), f"{name}: {text}"


def arguments(text, at):
    """The arguments of the call whose opening bracket is text[at], split at its own commas."""
    depth, start, out = 0, at + 1, []
    for i in range(at, len(text)):
        depth += text[i] in "([{"
        depth -= text[i] in ")]}"
        if depth == 0 or (depth == 1 and text[i] == ","):
            out.append(text[start:i].strip())
            start = i + 1
        if depth == 0:
            return out


def test_buffer_accesses_have_no_scalar_offset():
    """The end of a ring or of the drafted tokens is enforced by a buffer resource's size, and only the offset that a lane has of its
    own is sure to be compared with it: where the scalar offset is taken off the size, one that is larger leaves no end at all."""
    found = 0
    for path in sorted(glob.glob(os.path.join(CSRC, "*.h*p"))):
        text = re.sub(r"//[^\n]*", "", open(path).read())
        for m in re.finditer(r"__builtin_amdgcn_raw_buffer_(load|store)_\w+\(", text):
            args = arguments(text, m.end() - 1)
            assert len(args) == (4 if m.group(1) == "load" else 5), (path, args)
            assert args[-2] == "0", (os.path.basename(path), m.group(0), args)
            found += 1
    assert found >= 10
