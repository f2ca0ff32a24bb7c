"""Kernels of the built library for trees over a cache of 4 bits that are streamed: those that a call can reach.  bfloat16 goes through LDS from 17 rows on with up to 64 features, from 33 with up
to 128, from 65 above; a streaming kernel of 4, 2 and 1 shares of the keys is for up to 16, 32 and any number of rows."""
import os
import re

import pytest

LIB = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2009_13062_amd", "libnetfuse.so")


@pytest.mark.parametrize("kind,D,shares", [("t", 64, {4}), ("t", 128, {4, 2}), ("t", 256, {4, 2, 1}), ("f", 64, {4, 2, 1}), ("f", 128, {4, 2, 1}), ("f", 256, {4, 2, 1})])
def test_streaming_instances_are_reached(kind, D, shares):
    if not os.path.exists(LIB):
        import sys
        sys.path.insert(0, os.path.dirname(os.path.dirname(LIB)))
        import __graft_entry__ as g
        g.build()
    with open(LIB, "rb") as f:
        # <type, D, row blocks, shares, tree, 4 bits, exactly D features, up to 4 rows>
        found = set(re.findall(rb"decoder_stream_kernelI%sLi%dELi1ELi(\d)ELb1ELb1ELb([01])ELb([01])E" % (kind.encode(), D), f.read()))
    want = {(b"%d" % n, exact, b"0") for n in shares for exact in (b"0", b"1")} | ({(b"4", exact, b"1") for exact in (b"0", b"1")} if D <= 128 else set())
    assert found == want
