"""Wait states that the instruction set leaves to the program: the check of the library's code, on short sequences and on the library itself."""
import pytest

from paper_2504_20039_amd import check_isa

LOAD = "global_load_lds_dwordx4 v1, s[8:9]"


@pytest.mark.parametrize("between,missing", [([], 1), (["s_nop 0"], 0), (["v_add_u32_e32 v2, s3, v4"], 0)])
@pytest.mark.parametrize("load", [LOAD, "global_load_lds_dwordx4 v[2:3], off nt", "buffer_load_dwordx4 v1, s[4:7], 0 offen lds"])
@pytest.mark.parametrize("write", ["s_mov_b32 m0, s33", "s_add_i32 m0, s4, 0x400"])
def test_a_load_behind_a_write_of_m0(between, missing, load, write):
    found = check_isa.missing_waits(["_Z1kv:", write, *between, load])
    assert len(found) == missing and all("_Z1kv" in x for x in found)


def test_loads_that_do_not_read_m0():
    assert not check_isa.missing_waits(["s_mov_b32 m0, s33", "global_load_dwordx4 v[0:3], v1, s[8:9]"])
    assert not check_isa.missing_waits(["s_mov_b32 s0, m0", LOAD])
    assert not check_isa.missing_waits(["s_mov_b32 m0, s33 // 000000002EF4: BEFC0021", "s_endpgm", "0000000000001900 <_Z1kv>:", LOAD])


def test_the_library_keeps_them():
    import paper_2504_20039_amd as aj
    lines = check_isa.disassemble(aj.library_path())
    assert sum("global_load_lds_dwordx4" in x for x in lines) > 1000      # (the code was found)
    assert not check_isa.missing_waits(lines)
