"""Every access through a buffer descriptor has its whole offset where the descriptor's size is checked against it: in the vector register (or the instruction), not in the scalar one.

A row that is not there is left out by the size alone.  LLVM documents the scalar offset of raw buffer accesses as excluded from that check, and the hardware's manuals as taken off the size, which wraps where it is the larger."""
import os
import re

import pytest

import barriers

SCALAR = re.compile(r",\s*(s\d+|s\[\d+:\d+\]|m0|ttmp\d+|vcc_lo|vcc_hi|0x[0-9a-f]+|-?\d+(?:\.\d+)?)(?:\s+(?:offen|idxen|offset:\d+|nt|sc0|sc1|lds))*\s*$")


def unchecked(code):
    """[(address, instruction)] of buffer accesses with a scalar offset that is not zero."""
    bad = []
    for at, op, args, _ in code:
        if op.startswith("buffer_") and not op.startswith(("buffer_wbl2", "buffer_inv")):
            m = SCALAR.search("," + args)
            assert m, (op, args)
            if m.group(1) != "0":
                bad.append((at, op + " " + args))
    return bad


@pytest.mark.parametrize("args,fine", [("v10, v2, s[8:11], 0 offen", True), ("v10, v2, s[8:11], 0 offen offset:64 nt", True), ("v10, v2, s[8:11], s12 offen nt", False), ("v10, off, s[8:11], s12", False),
                                       ("v[1:4], off, s[8:11], 0", True), ("v6, s[4:7], 0 offen lds", True), ("v10, v2, s[8:11], 64 offen", False)])
def test_what_is_found(args, fine):
    assert (unchecked([(0, "buffer_load_dword", args, None)]) == []) == fine


def test_every_buffer_access_of_the_library():
    from paper_2604_04921_amd import binding as B
    assert os.path.exists(B.LIB_PATH), "libtri.so is not built"
    kernels = barriers.functions(B.LIB_PATH)
    assert sum(op.startswith("buffer_load") for code in kernels.values() for _, op, _, _ in code) > 1000
    assert not {k: b for k, b in ((k, unchecked(code)) for k, code in kernels.items()) if b}
