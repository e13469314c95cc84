"""No kernel of the built library reaches a barrier with LDS writes, or loads into LDS, that have not been waited for."""
import os

import pytest

import barriers

LOOP = """
0000000000001000 <kernel>:
	s_mov_b32 s0, 0                                            // 000000001000: 00000000
	s_barrier                                                  // 000000001004: 00000000
	ds_write_b32 v0, v1                                        // 000000001008: 00000000
	ds_bpermute_b32 v2, v3, v4                                 // 00000000100C: 00000000
	%s                                                         // 000000001010: 00000000
	s_cbranch_scc1 65533                                       // 000000001014: 00000000 <kernel+0x4>
	s_endpgm                                                   // 000000001018: 00000000
"""


@pytest.mark.parametrize("instruction,fine", [("s_nop 0", False), ("s_waitcnt vmcnt(0)", False), ("s_waitcnt lgkmcnt(2)", False), ("s_waitcnt lgkmcnt(1)", True), ("s_waitcnt vmcnt(0) lgkmcnt(0)", True),
                                              ("s_load_dword s1, s[2:3], 0x0", False), ("buffer_load_dwordx4 v6, s[4:7], 0 offen lds", False)])
def test_what_is_found(instruction, fine):
    """A write on the way round a loop, behind whose barrier it is read."""
    code = barriers.parse(LOOP % instruction)["kernel"]
    assert [op for _, op, _, _ in code][1] == "s_barrier" and code[5][3] == 0x1004
    assert (barriers.unwaited(code) == []) == fine


def test_scalar_loads_come_in_any_order():
    text = LOOP % "s_load_dword s1, s[2:3], 0x0"
    for wait, fine in (("lgkmcnt(1)", False), ("lgkmcnt(0)", True)):
        code = barriers.parse(text)["kernel"]
        code.insert(5, (0x1012, "s_waitcnt", wait, None))
        assert (barriers.unwaited(code) == []) == fine


def test_every_barrier_of_the_library():
    from paper_2604_04921_amd import binding as B
    assert os.path.exists(B.LIB_PATH), "libtri.so is not built"
    kernels = barriers.functions(B.LIB_PATH)
    assert sum("attend_tile_kernel" in k for k in kernels) >= 12 and sum(op == "s_barrier" for code in kernels.values() for _, op, _, _ in code) > 100
    bad = {k: b for k, b in ((k, barriers.unwaited(code)) for k, code in kernels.items()) if b}
    assert not bad
