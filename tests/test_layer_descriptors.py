"""Loads written as inline assembly read buffer descriptors whose registers a vector instruction may have written just
before: five cycles have to lie between, which the compiler counts for its own loads only.  Wherever the sources make a
descriptor it has to go through a pause that names it, so that neither the compiler nor a later change comes between."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_16907_amd", "csrc")
FILES = [f for f in sorted(glob.glob(os.path.join(CSRC, "*"))) if "buffer_load" in open(f).read()]


def functions(text):
    """(name, body) of what is defined with braces on lines of their own indentation."""
    for at in re.finditer(r"^( *)(?:template.*>\n\1)?__device__ [^;{]*?(\w+)\([^;{]*\)(?: const)? \{\n", text, re.M):
        end = re.compile(r"^%s\}" % at.group(1), re.M).search(text, at.end())
        yield at.group(2), text[at.end():end.start()]


@pytest.mark.parametrize("file", FILES, ids=os.path.basename)
def test_descriptors_are_settled(file):
    text = open(file).read()
    makers = [(name, body) for name, body in functions(text) if re.search(r"\bd\[0\] = __builtin_amdgcn_readfirstlane", body)]
    for name, body in makers:
        after = body[body.rindex("readfirstlane"):]
        if re.search(r'asm volatile\("s_nop 4" : "\+s"\(d\)\);', after):
            continue
        # it is left to the callers: each use is followed by settle() on the same object
        uses = re.findall(r"(\w+)\.%s\((.*)" % name, text)
        assert uses, (name, "has no pause")
        for of, rest in uses:
            assert "%s.settle()" % of in rest or "if constexpr (!inner) sp.settle(), sq.settle();" in text, (name, of, rest)


def test_both_makers_are_seen():
    found = {name for f in FILES for name, body in functions(open(f).read()) if re.search(r"\bd\[0\] = __builtin_amdgcn_readfirstlane", body)}
    assert {"descriptor", "open"} <= found
